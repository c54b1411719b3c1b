// Appending to a paged K/V cache for gfx950: new keys are rotated by their positions and written into the pages that the
// block table names, values are copied there, queries are rotated on the way.
//
// Rotation: for a pair (a, b) of elements of a head and the angle of (position, pair)
//     a' = a cos - b sin,   b' = b cos + a sin
// in 32 bits, rounded once to the element type; cosines and sines come from a table by position.  A pair is (i, i + rot/2)
// or, interleaved, (2i, 2i + 1), i < rot/2.
//
// What bounds it: memory (each element is read once and written once; a fused projection's row of 32 + 2 * 8 heads of width
// 128 is 12 KiB, the table's row 512 bytes).  So WPT waves take one token: their lanes are (row, 16 elements), a row being a
// query, key or value head, and walk the rows with the same 16 elements: the table's values stay in registers for all of
// the token's heads.  kRows rows are in flight together, and they are requested before the position is known, which the
// table's row and the page wait for (one token of four sequences 5.2 / 3.4 us, of 256 5.7 / 3.9 before and since).  A 32K prompt of 32
// heads over 8: 171 us, 5.2 TB/s; a large copy moves 4.9.
#include "bsfa_dev.h"

namespace bsfa {

// Rows a lane has in flight (1 / 2 / 3 / 6, us: a 32K prompt 176 / 172 / 173 / 170; 6 prompts of 700 to 4000 tokens of width 64
// 14.9 / 14.7 / 15.9 / 18.9, whose registers leave room for fewer waves).
constexpr int kRows = 2;
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int D, bool F16, bool INTERLEAVED, int WPT>
__global__ void __launch_bounds__(256) append_kernel(const AppendParams p)
{
    typedef typename Elem<F16>::T el;
    typedef typename Elem<F16>::x8 el8;
    constexpr int TPR = D / 16;                          // lanes of a row
    constexpr int RPW = 64 * WPT / TPR;                  // rows at a time
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & (64 * WPT - 1);
    const uint32_t tok = blockIdx.x * (4 / WPT) + wave / WPT;
    if (tok >= (uint32_t)p.batch * (uint32_t)p.seqlen) return;
    const int b = (int)p.div_seqlen.of(tok), i = (int)(tok - (uint32_t)b * (uint32_t)p.seqlen);
    if (p.seqlens && i >= p.seqlens[b]) return;
    const int start = p.start[b];

    // this lane's 16 elements of every row: two runs of 8, the halves of 8 pairs (or, interleaved and behind the rotated
    // elements, 16 adjacent ones)
    const int part = lane % TPR;
    const bool turns = part * 16 < p.rot;
    const int at0 = INTERLEAVED || !turns ? part * 16 : part * 8;
    const int at1 = INTERLEAVED || !turns ? at0 + 8 : at0 + p.rot / 2;
    const int hq = p.q ? p.hq : 0, rows = hq + 2 * p.hkv;
    el8 lo[kRows], hi[kRows];
    auto load = [&](int r0) {
#pragma unroll
        for (int n = 0; n < kRows; ++n) {
            const int r = r0 + n * RPW, h = r - hq;
            if (r >= rows) break;
            const uint16_t *src = r < hq ? p.q + b * p.qsb + i * p.qsn + r * p.qsh
                                : h < p.hkv ? p.k + b * p.ksb + i * p.ksn + h * p.ksh : p.v + b * p.vsb + i * p.vsn + (h - p.hkv) * p.vsh;
            const bool value = h >= p.hkv;               // (a value's runs are adjacent)
            lo[n] = *reinterpret_cast<const el8 *>(src + (value ? part * 16 : at0));
            hi[n] = *reinterpret_cast<const el8 *>(src + (value ? part * 16 + 8 : at1));
        }
    };
    load(lane / TPR);

    const int64_t pos = (int64_t)start + i;
    if (pos < 0 || pos >= (int64_t)p.table_pages << p.pages.page_log2) return;           // has no place in the table
    const int page = p.table[b * p.tsb + (pos >> p.pages.page_log2)];
    const bool stored = page >= 0 && page < p.pages.n_pages;
    const int64_t place = pos & ((1 << p.pages.page_log2) - 1);
    f32x4 cs[2], sn[2];                                  // of the pairs that begin at at0 (interleaved: half of it)
    if (turns) {
        const float *t = p.cos_sin + pos * p.rot + part * 8;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            cs[e] = *reinterpret_cast<const f32x4 *>(t + 4 * e);
            sn[e] = *reinterpret_cast<const f32x4 *>(t + p.rot / 2 + 4 * e);
        }
    }
    for (int r0 = lane / TPR; r0 < rows;) {
#pragma unroll
        for (int n = 0; n < kRows; ++n) {
            const int r = r0 + n * RPW, h = r - hq;
            if (r >= rows) break;
            if (h >= p.hkv) {
                if (stored) {
                    uint16_t *dst = p.v_cache + page * p.pages.vsp + place * p.pages.vsn + (h - p.hkv) * p.pages.vsh + part * 16;
                    *reinterpret_cast<el8 *>(dst) = lo[n];
                    *reinterpret_cast<el8 *>(dst + 8) = hi[n];
                }
                continue;
            }
            if (turns) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const auto turn = [&](el &x, el &y, int pair) {
                        const float a = (float)x, c = (float)y, co = cs[pair >> 2][pair & 3], si = sn[pair >> 2][pair & 3];
                        x = (el)(a * co - c * si);
                        y = (el)(c * co + a * si);
                    };
                    el x, y;
                    if constexpr (INTERLEAVED) {
                        x = e < 4 ? lo[n][2 * e] : hi[n][2 * e - 8];
                        y = e < 4 ? lo[n][2 * e + 1] : hi[n][2 * e - 7];
                        turn(x, y, e);
                        if (e < 4) lo[n][2 * e] = x, lo[n][2 * e + 1] = y;
                        else hi[n][2 * e - 8] = x, hi[n][2 * e - 7] = y;
                    } else {
                        x = lo[n][e];
                        y = hi[n][e];
                        turn(x, y, e);
                        lo[n][e] = x;
                        hi[n][e] = y;
                    }
                }
            }
            uint16_t *dst[2] = {nullptr, nullptr};
            if (r < hq) dst[0] = p.q_out + b * p.qosb + i * p.qosn + r * p.qosh;
            else {
                if (stored) dst[0] = p.k_cache + page * p.pages.ksp + place * p.pages.ksn + h * p.pages.ksh;
                if (p.k_out) dst[1] = p.k_out + b * p.kosb + i * p.kosn + h * p.kosh;
            }
#pragma unroll
            for (int o = 0; o < 2; ++o)
                if (dst[o]) {
                    *reinterpret_cast<el8 *>(dst[o] + at0) = lo[n];
                    *reinterpret_cast<el8 *>(dst[o] + at1) = hi[n];
                }
        }
        r0 += RPW * kRows;
        if (r0 < rows) load(r0);
    }
}

template <int D, bool F16, int WPT> static void launch(const AppendParams &p, hipStream_t stream)
{
    const unsigned grid = (unsigned)(((int64_t)p.batch * p.seqlen * WPT + 3) / 4);
    if (p.interleaved) append_kernel<D, F16, true, WPT><<<grid, 256, 0, stream>>>(p);
    else append_kernel<D, F16, false, WPT><<<grid, 256, 0, stream>>>(p);
}
template <int D, bool F16> static void launch(const AppendParams &p, hipStream_t stream)
{
    // (one wave / four, us: 512 tokens 6.3 / 5.1, 2048 11.4 / 11.2, 4096 19.0 / 19.1)
    if ((int64_t)p.batch * p.seqlen <= 2048) launch<D, F16, 4>(p, stream);
    else launch<D, F16, 1>(p, stream);
}

hipError_t launch_append(const AppendParams &params, int head_dim, bool f16, hipStream_t stream)
{
    AppendParams p = params;
    p.div_seqlen = fast_div((uint32_t)p.seqlen);
    if (head_dim == 128) f16 ? launch<128, true>(p, stream) : launch<128, false>(p, stream);
    else if (head_dim == 64) f16 ? launch<64, true>(p, stream) : launch<64, false>(p, stream);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace bsfa
