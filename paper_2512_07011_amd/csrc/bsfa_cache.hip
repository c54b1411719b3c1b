// Appending to a paged K/V cache for gfx950: new keys are rotated by their positions and written into the pages that the
// block table names, values are copied there, queries are rotated on the way.
//
// Rotation: for a pair (a, b) of elements of a head and the angle of (position, pair)
//     a' = a cos - b sin,   b' = b cos + a sin
// in 32 bits, rounded once to the element type; cosines and sines come from a table by position.  A pair is (i, i + rot/2)
// or, interleaved, (2i, 2i + 1), i < rot/2.
//
// What bounds it: memory (each element is read once and written once; a fused projection's row of 32 + 2 * 8 heads of width
// 128 is 12 KiB, the table's row 512 bytes).  So a wave takes one token: its lanes are (row, 16 elements), a row being a
// query, key or value head, and walk the rows with the same 16 elements: the table's values stay in registers for all of
// the token's heads.  Loads of kRows rows are in flight together, and they do not wait for the position or the page.
#include "bsfa_dev.h"

namespace bsfa {

constexpr int kRows = 3;             // rows a lane has in flight

template <int D, bool F16, bool INTERLEAVED>
__global__ void __launch_bounds__(256) append_kernel(const AppendParams p)
{
    typedef typename Elem<F16>::T el;
    typedef typename Elem<F16>::x8 el8;
    constexpr int TPR = D / 16;                          // lanes of a row
    constexpr int RPW = 64 / TPR;                        // rows of a wave at a time
    const int lane = threadIdx.x & 63;
    const uint32_t tok = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (tok >= (uint32_t)p.batch * (uint32_t)p.seqlen) return;
    const int b = (int)p.div_seqlen.of(tok), i = (int)(tok - (uint32_t)b * (uint32_t)p.seqlen);
    if (p.seqlens && i >= p.seqlens[b]) return;
    const int64_t pos = (int64_t)p.start[b] + i;
    if (pos < 0 || pos >= (int64_t)p.table_pages << p.pages.page_log2) return;           // has no place in the table
    const int page = p.table[b * p.tsb + (pos >> p.pages.page_log2)];
    const bool stored = page >= 0 && page < p.pages.n_pages;
    const int64_t place = pos & ((1 << p.pages.page_log2) - 1);

    // this lane's 16 elements of every row: two runs of 8, the halves of 8 pairs (or, interleaved and behind the rotated
    // elements, 16 adjacent ones)
    const int part = lane % TPR;
    const bool turns = part * 16 < p.rot;
    const int at0 = INTERLEAVED || !turns ? part * 16 : part * 8;
    const int at1 = INTERLEAVED || !turns ? at0 + 8 : at0 + p.rot / 2;
    float cs[8], sn[8];                                  // of the pairs that begin at at0 (interleaved: half of it)
    if (turns) {
        const float *t = p.cos_sin + pos * p.rot + part * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            cs[e] = t[e];
            sn[e] = t[p.rot / 2 + e];
        }
    }

    const int hq = p.q ? p.hq : 0, rows = hq + 2 * p.hkv;
    for (int r0 = lane / TPR; r0 < rows; r0 += RPW * kRows) {
        el8 lo[kRows], hi[kRows];
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
                    if constexpr (INTERLEAVED) {
                        if (e & 1) continue;
                        const float a = (float)lo[n][e], c = (float)lo[n][e + 1], a2 = (float)hi[n][e], c2 = (float)hi[n][e + 1];
                        lo[n][e] = (el)(a * cs[e / 2] - c * sn[e / 2]);
                        lo[n][e + 1] = (el)(c * cs[e / 2] + a * sn[e / 2]);
                        hi[n][e] = (el)(a2 * cs[4 + e / 2] - c2 * sn[4 + e / 2]);
                        hi[n][e + 1] = (el)(c2 * cs[4 + e / 2] + a2 * sn[4 + e / 2]);
                    } else {
                        const float a = (float)lo[n][e], c = (float)hi[n][e];
                        lo[n][e] = (el)(a * cs[e] - c * sn[e]);
                        hi[n][e] = (el)(c * cs[e] + a * sn[e]);
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
    }
}

template <int D, bool F16> static void launch(const AppendParams &p, unsigned grid, hipStream_t stream)
{
    if (p.interleaved) append_kernel<D, F16, true><<<grid, 256, 0, stream>>>(p);
    else append_kernel<D, F16, false><<<grid, 256, 0, stream>>>(p);
}

hipError_t launch_append(const AppendParams &params, int head_dim, bool f16, hipStream_t stream)
{
    AppendParams p = params;
    p.div_seqlen = fast_div((uint32_t)p.seqlen);
    const unsigned grid = (unsigned)(((int64_t)p.batch * p.seqlen + 3) / 4);
    if (head_dim == 128) f16 ? launch<128, true>(p, grid, stream) : launch<128, false>(p, grid, stream);
    else if (head_dim == 64) f16 ? launch<64, true>(p, grid, stream) : launch<64, false>(p, grid, stream);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace bsfa
