// Attention of new tokens over a paged K/V cache for gfx950, wave64, bf16 or fp16 MFMA:
//     o_i = sum_t softmax_t(q_i k_t / sqrt(d)) v_t
// over the tokens t that query i sees: those its sequence has in its own pages (causal: up to i's own place) and those of a
// prefix that all sequences share.  One pass over the keys with a running maximum m, normaliser l and unscaled accumulator
// O; ranges of keys are worked on apart and joined by
//     m = max m_x,  l = sum l_x 2^(m_x - m),  O = sum O_x 2^(m_x - m)          (log2 units).
// The (query token, query head) pairs that read one KV head are the rows of a unit: one sequence's, or for the prefix
// everybody's.
#include "bsfa_dev.h"

#include <algorithm>

namespace bsfa {

typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 mfma32(bf16x8_t a, bf16x8_t b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma32(f16x8_t a, f16x8_t b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

constexpr float kNone = -3.0e38f;    // running maximum of a row that has seen no key: finite, below any score
constexpr int kSub = 16;             // keys that lie in one page whatever its size

struct Launch {
    PagedParams p;
    int extra;                       // > 0: own tokens are cut into ranges, batch + extra at most; 0: one range a sequence
    int rows;                        // rows of a unit
    int groups;                      // row groups of a unit, one to a workgroup
    int chunk;                       // keys of a range of the prefix
    int parts;                       // ranges of the prefix
    float *own_o, *prefix_o;         // unscaled results of ranges: [range][hkv][rows][d] ...
    float2 *own_ml, *prefix_ml;      // ... and their (m, l)
    bool direct;                     // a sequence in one range is written to out at once
};

// ---- ranges of a batch's own tokens ---------------------------------------------------------------
// Every range is `chunk` tokens or less; chunk follows from the lengths on the device, so that a captured launch stays
// even as sequences grow: with chunk >= total / extra there are at most batch + extra ranges.
struct Range {
    int b, part, parts, first, len, chunk;               // sequence, which range of how many; number of ranges before the sequence's
};

__device__ __forceinline__ int length_of(const PagedParams &p, int b) { return min(max(p.cache_lens[b], 0), p.max_len); }
__device__ __forceinline__ int queries_of(const PagedParams &p, int b) { return p.q_lens ? min(max(p.q_lens[b], 0), p.seqlen) : p.seqlen; }

// Counts the ranges off, in every wave alike: the sequence that holds range x (by_range) or the sequence x.
template <bool BY_RANGE> __device__ __forceinline__ bool find_range(const Launch &a, int x, Range &r)
{
    const PagedParams &p = a.p;
    r.first = 0;
    r.part = 0;
    r.parts = 1;
    r.b = x;
    r.chunk = 0x7fffffff;
    if (a.extra == 0) {
        r.first = x;
        r.len = __builtin_amdgcn_readfirstlane(length_of(p, x));
        return true;
    }
    const int lane = threadIdx.x & 63;
    unsigned long long total = 0;
    for (int b = lane; b < p.batch; b += 64) total += (unsigned)length_of(p, b);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) total += __shfl_xor(total, s);
    const unsigned long long even = (total + a.extra - 1) / (unsigned)a.extra;
    r.chunk = (int)min(max((even + 127) & ~127ull, 128ull), 0x7fffff80ull);
    r.chunk = __builtin_amdgcn_readfirstlane(r.chunk);
    int before = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
        const int b = b0 + lane, len = b < p.batch ? length_of(p, b) : 0;
        const int n = b >= p.batch ? 0 : len > 0 ? (len - 1) / r.chunk + 1 : 1;
        int upto = n;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int y = __shfl_up(upto, s);
            upto += lane >= s ? y : 0;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (BY_RANGE ? x < before + all : x < b0 + 64) {
            const int l = BY_RANGE ? __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + upto > x)) : x - b0;
            r.b = b0 + l;
            r.parts = __builtin_amdgcn_readlane(n, l);
            r.first = before + __builtin_amdgcn_readlane(upto, l) - r.parts;
            r.len = __builtin_amdgcn_readlane(len, l);
            r.part = x - r.first;
            return true;
        }
        before += all;
    }
    return false;
}

// ---- tiles of keys in LDS ---------------------------------------------------------------------------
// Kept as sub-blocks of 16 keys, rows of 2 D bytes, without gaps (a direct copy's LDS side is linear).  The 16-byte chunks
// of a row are permuted among themselves, c -> c ^ swizzle(row), on the global side of the copy, so that 16 rows read at
// one chunk (K) or at a pair of chunks (V) use all banks evenly.
template <int D> __device__ __forceinline__ int swizzle(int row) { return D == 128 ? row & 15 : ((row >> 1) & 3) * 2 + ((row >> 3) & 1); }

template <int D> struct SubBlock {
    static constexpr int BYTES = kSub * D * 2;
    static constexpr int UNITS = BYTES / kUnit;          // direct copies of a wave
    static constexpr int ROWS = kSub / UNITS;            // rows of a copy
    // byte offsets of a lane's 16 bytes of every unit, rows `stride` elements apart
    __device__ __forceinline__ static void offsets(uint32_t (&off)[UNITS], int lane, int64_t stride)
    {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int row = u * ROWS + lane / (D / 8);
            off[u] = (uint32_t)(row * (int)stride + ((lane % (D / 8)) ^ swizzle<D>(row)) * 8) * 2u;
        }
    }
    // of the sub-block whose first row is at `src`; of its rows only `n` exist, the others become 0
    __device__ __forceinline__ static i32x4 descriptor(const uint16_t *src, int n, int64_t stride)
    {
        const uint64_t at = reinterpret_cast<uint64_t>(src);
        const i32x4 rsrc = {(int)(uint32_t)at, (int)((uint32_t)(at >> 32) & 0xffffu), n > 0 ? ((n - 1) * (int)stride + D) * 2 : 0, 0x00020000};
        asm volatile("s_nop 3" : : "s"(rsrc));           // (a descriptor from a vector instruction is read 5 states later at the earliest)
        return rsrc;
    }
    // requests unit U into the sub-block's place `dst`, which is uniform
    template <int U> __device__ __forceinline__ static void unit(i32x4 rsrc, uint32_t off, uint32_t dst)
    {
        asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %3, 0 offen lds"
                     : : "v"(off), "s"(dst), "n"(U * kUnit), "s"(rsrc) : "memory", "m0", "scc");
    }
    __device__ __forceinline__ static void copy(const uint16_t *src, int n, int64_t stride, const uint32_t (&off)[UNITS], uint32_t lds)
    {
        const i32x4 rsrc = descriptor(src, n, stride);
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds);
        static_for<UNITS>([&](auto u) { unit<decltype(u)::value>(rsrc, off[decltype(u)::value], dst); });
    }
};

// the page table is read through the scalar cache, which neither the copies' counter nor their waits know of
__device__ __forceinline__ int page_id(const int32_t *table, int token, int log2, int last)
{
    return ((const __attribute__((address_space(4))) int32_t *)table)[min(token >> log2, last)];
}

// max over lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quad_max(float x)
{
    float a = x, b;
    asm volatile("v_mov_b32 %1, %0\n\ts_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1\n\tv_max_f32 %0, %0, %1" : "+v"(a), "=&v"(b));
    return pair_max(a);
}

__device__ __forceinline__ float quad_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Where a row's query and result lie.
struct Row {
    int b, i, h;                                         // sequence, new token, query head
    bool stored;                                         // there is such a row
};
template <bool PREFIX> __device__ __forceinline__ Row row_of(const Launch &a, int r, int b, int hk)
{
    const PagedParams &p = a.p;
    const int rr = min(r, a.rows - 1), t = rr / p.group;
    Row x;
    x.b = PREFIX ? t / p.seqlen : b;
    x.i = PREFIX ? t - x.b * p.seqlen : t;
    x.h = hk * p.group + rr - t * p.group;
    x.stored = r < a.rows;
    return x;
}

// ---- few rows: keys streamed once ---------------------------------------------------------------------
// A workgroup is NW waves on 16 * NRT rows of one unit and one range of keys.  Every wave takes tiles of 32 keys of its own
// (the wave-th of every NW), with a ring of kStages tiles in LDS that only it reads: no barrier until the waves' results
// are joined at the end.
//   S^T = K Q^T   16x16x32 MFMA, fp32; column = row of the unit, so that a row's scores lie in four lanes
//   O^T += V^T P^T, V^T through the transposing LDS read; the accumulator layout of S^T is the operand layout of P^T up to
//   an order of the keys that V's reads share, so P never leaves the registers.
// Rounded: P to the element type for the second product (its operands have it); l sums the unrounded fp32 values.
constexpr int kStages = 2;

template <int D, int NW, int NRT, bool F16, bool PREFIX>
__global__ void __launch_bounds__(NW * 64, 1) paged_stream_kernel(const Launch a)
{
    typedef typename Elem<F16>::T el;
    typedef typename Elem<F16>::x8 el8;
    typedef SubBlock<D> SB;
    constexpr int KI = D / 32;                           // MFMAs of a score tile
    constexpr int DB = D / 16;                           // 16-row blocks of O^T
    constexpr int STAGE = 4 * SB::BYTES;                 // K of two sub-blocks, V of two
    constexpr int PER_STAGE = 4 * SB::UNITS;             // copies
    constexpr int OPITCH = D + 4;                        // floats of a row where the waves' results are joined
    static_assert(NW * kSub * OPITCH * 4 <= NW * kStages * STAGE, "joining fits the ring");
    __shared__ __attribute__((aligned(1024))) unsigned char ring[NW * kStages * STAGE];
    __shared__ float red_m[NW][kSub * NRT], red_l[NW][kSub * NRT];

    const PagedParams &p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hk = blockIdx.x % p.hkv, w = blockIdx.x / p.hkv;
    const int rg = w % a.groups, x = w / a.groups;
    Range r;
    int qn = p.seqlen, k0, k1;
    if constexpr (PREFIX) {
        r.b = 0, r.part = x, r.parts = a.parts, r.first = 0, r.len = p.prefix;
        k0 = x * a.chunk;
        k1 = min(p.prefix, k0 + a.chunk);
    } else {
        if (!find_range<true>(a, x, r)) return;
        qn = __builtin_amdgcn_readfirstlane(queries_of(p, r.b));
        k0 = r.part * r.chunk;                           // (part 0 where chunk is the largest number)
        k1 = (int)min((int64_t)r.len, (int64_t)k0 + r.chunk);
    }
    const int row0 = rg * kSub * NRT;
    const int n16 = lane & 15, quad = lane >> 4;
    int sees[NRT];                                       // keys below it are visible to this lane's row
    int all_see = k1;                                    // ... to every row
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        sees[t] = k1;
        if (!PREFIX && p.causal) sees[t] = min(k1, r.len - qn + row_of<PREFIX>(a, row0 + t * kSub + n16, r.b, hk).i + 1);
    }
    if (!PREFIX && p.causal) {
        all_see = min(k1, r.len - qn + row0 / p.group + 1);
        k1 = min(k1, r.len - qn + min(row0 + kSub * NRT - 1, a.rows - 1) / p.group + 1);      // keys that some row sees
    }

    const int32_t *table = PREFIX ? p.prefix_table : p.table + r.b * p.tsb;
    const int last_page = max(k1 - 1, 0) >> p.pages.page_log2, in_page = (1 << p.pages.page_log2) - 1;
    el8 q[NRT][KI];
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        const Row y = row_of<PREFIX>(a, row0 + t * kSub + n16, r.b, hk);
        const uint16_t *src = p.q + y.b * p.qsb + y.i * p.qsn + y.h * p.qsh + quad * 8;
#pragma unroll
        for (int i = 0; i < KI; ++i) q[t][i] = *reinterpret_cast<const el8 *>(src + 32 * i);
    }
    uint32_t koff[SB::UNITS], voff[SB::UNITS];
    SB::offsets(koff, lane, p.pages.ksn);
    SB::offsets(voff, lane, p.pages.vsn);
    const uint32_t mine = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) unsigned char *)ring) + wave * kStages * STAGE;
    const uint16_t *const kh = p.k_cache + hk * p.pages.ksh, *const vh = p.v_cache + hk * p.pages.vsh;

    struct Ids { int id[2]; };
    auto ids_of = [&](int key) {                         // pages of a tile's two sub-blocks
        Ids y;
        y.id[0] = page_id(table, key, p.pages.page_log2, last_page);
        y.id[1] = page_id(table, key + kSub, p.pages.page_log2, last_page);
        return y;
    };
    // keys of a sub-block that exist: none where it lies behind the range or its page is none of the cache's
    auto exist = [&](int key, int id) { return __builtin_amdgcn_readfirstlane((unsigned)id < (unsigned)p.pages.n_pages ? min(max(k1 - key, 0), kSub) : 0); };
    auto request = [&](int key, const Ids &ids, uint32_t at) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int n = exist(key + s * kSub, ids.id[s]);
            const int64_t id = n > 0 ? ids.id[s] : 0, place = (key + s * kSub) & in_page;
            SB::copy(kh + id * p.pages.ksp + place * p.pages.ksn, n, p.pages.ksn, koff, at + s * SB::BYTES);
            SB::copy(vh + id * p.pages.vsp + place * p.pages.vsn, n, p.pages.vsn, voff, at + (2 + s) * SB::BYTES);
        }
    };

    f32x4 o[NRT][DB];
    float m[NRT], l[NRT];
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        m[t] = kNone;
        l[t] = 0.f;
#pragma unroll
        for (int x = 0; x < DB; ++x) o[t][x] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // addresses of a lane's operands inside a sub-block.  K: key n16, elements 32 i + 8 quad .. + 7.  V: key
    // 4 quad + (n16 >> 2), elements 16 x + 4 (n16 & 3) .. + 3, which the read transposes within 16 lanes.
    uint32_t ka[KI], va[DB];
#pragma unroll
    for (int i = 0; i < KI; ++i) ka[i] = n16 * (D * 2) + (((4 * i + quad) ^ swizzle<D>(n16)) * 16);
    const int vrow = 4 * quad + (n16 >> 2);
#pragma unroll
    for (int x = 0; x < DB; ++x) va[x] = vrow * (D * 2) + (((2 * x + ((n16 >> 1) & 1)) ^ swizzle<D>(vrow)) * 16) + (n16 & 1) * 8 + 2 * SB::BYTES;

    constexpr int STEP = 32 * NW;
    int key = k0 + 32 * wave;
    Ids now = ids_of(key), next = ids_of(key + STEP);
    // the queries arrive before the copies are requested: a wait for them would wait for the copies, too
#pragma unroll
    for (int t = 0; t < NRT; ++t)
#pragma unroll
        for (int i = 0; i < KI; ++i) asm volatile("" : "+v"(q[t][i]));
    request(key, now, mine);
    request(key + STEP, next, mine + STAGE);
    Ids after = ids_of(key + 2 * STEP);
    uint32_t at = mine;
    for (; key < k1; key += STEP) {
        wait_vmcnt<PER_STAGE>();
        asm volatile("" : : : "memory");
        f32x4 s[NRT][2];
#pragma unroll
        for (int t = 0; t < NRT; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < KI; ++i) {
                const el8 kk = *LDS_PTR(const el8, at + ka[i] + kb * SB::BYTES);
#pragma unroll
                for (int t = 0; t < NRT; ++t) s[t][kb] = mfma32(kk, q[t][i], s[t][kb]);
            }
        const int n0 = exist(key, now.id[0]), n1 = exist(key + kSub, now.id[1]);
        if (n0 + n1 < 32 || key + 32 > all_see) {
#pragma unroll
            for (int t = 0; t < NRT; ++t)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int y = 4 * quad + e;
                        if (y >= (kb ? n1 : n0) || key + kb * kSub + y >= sees[t]) s[t][kb][e] = -INFINITY;
                    }
        }
        el8 pr[NRT];
#pragma unroll
        for (int t = 0; t < NRT; ++t) {
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][kb][e]);
            mx = fmaxf(m[t], quad_max(mx) * p.scale_log2);
            if (__builtin_amdgcn_ballot_w64(mx > m[t])) {
                const float f = __builtin_amdgcn_exp2f(m[t] - mx);
                l[t] *= f;
#pragma unroll
                for (int x = 0; x < DB; ++x) o[t][x] *= f;
                m[t] = mx;
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = __builtin_amdgcn_exp2f(fmaf(s[t][kb][e], p.scale_log2, -m[t]));
                    l[t] += y;
                    pr[t][4 * kb + e] = (el)y;
                }
        }
#pragma unroll
        for (int x = 0; x < DB; ++x) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + va[x]));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + va[x] + SB::BYTES));
            const el8 vv = __builtin_bit_cast(el8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int t = 0; t < NRT; ++t) o[t][x] = mfma32(vv, pr[t], o[t][x]);
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0): this tile has been read
        asm volatile("" : : : "memory");
        request(key + 2 * STEP, after, at);
        now = next;
        next = after;
        after = ids_of(key + 3 * STEP);
        at ^= mine ^ (mine + STAGE);
    }

    // ---- the waves' results joined, 16 rows at a time --------------------------------------------------
    wait_vmcnt<0>();
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        l[t] = quad_sum(l[t]);
        if (quad == 0) {
            red_m[wave][t * kSub + n16] = m[t];
            red_l[wave][t * kSub + n16] = l[t];
        }
    }
    float *const ro = reinterpret_cast<float *>(ring);
    constexpr int TPR = NW * 64 / kSub, DPT = D / TPR;   // threads of a row, elements of a thread
    const int jr = threadIdx.x / TPR, jd = threadIdx.x % TPR * DPT;
    const bool direct = !PREFIX && a.direct && r.parts == 1;
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        __syncthreads();
#pragma unroll
        for (int x = 0; x < DB; ++x) *reinterpret_cast<f32x4 *>(ro + (wave * kSub + n16) * OPITCH + 16 * x + 4 * quad) = o[t][x];
        __syncthreads();
        const int row = row0 + t * kSub + jr;
        const Row y = row_of<PREFIX>(a, row, r.b, hk);
        float mm = kNone, ll = 0.f, oo[DPT];
#pragma unroll
        for (int v = 0; v < NW; ++v) mm = fmaxf(mm, red_m[v][t * kSub + jr]);
#pragma unroll
        for (int d = 0; d < DPT; ++d) oo[d] = 0.f;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const float f = __builtin_amdgcn_exp2f(red_m[v][t * kSub + jr] - mm);
            ll = fmaf(f, red_l[v][t * kSub + jr], ll);
#pragma unroll
            for (int d = 0; d < DPT; ++d) oo[d] = fmaf(f, ro[(v * kSub + jr) * OPITCH + jd + d], oo[d]);
        }
        if (!y.stored) continue;
        if (direct) {
            if (y.i >= qn) continue;
            const float f = ll > 0.f ? 1.f / ll : 0.f;   // (a row that sees nothing: 0)
            uint16_t *dst = p.out + y.b * p.osb + y.i * p.osn + y.h * p.osh + jd;
            typedef el elx __attribute__((ext_vector_type(DPT)));
            elx z;
#pragma unroll
            for (int d = 0; d < DPT; ++d) z[d] = (el)(oo[d] * f);
            *reinterpret_cast<elx *>(dst) = z;
            if (p.lse && jd == 0) p.lse[((int64_t)y.b * p.seqlen + y.i) * p.hq + y.h] = ll > 0.f ? 0.6931471805599453f * (mm + __builtin_amdgcn_logf(ll)) : -INFINITY;
        } else {
            const int64_t slot = ((int64_t)(PREFIX ? x : r.first + r.part) * p.hkv + hk) * a.rows + row;
            float *dst = (PREFIX ? a.prefix_o : a.own_o) + slot * D + jd;
#pragma unroll
            for (int d = 0; d < DPT; d += 4) *reinterpret_cast<f32x4 *>(dst + d) = f32x4{oo[d], oo[d + 1], oo[d + 2], oo[d + 3]};
            if (jd == 0) (PREFIX ? a.prefix_ml : a.own_ml)[slot] = make_float2(mm, ll);
        }
    }
}

// ---- many rows: keys shared by a workgroup's waves ------------------------------------------------------
// Four waves of 32 rows on tiles of 64 keys, K and V in two LDS slots each; a wave copies the sub-block of its number.
//   S^T = K Q^T, O^T += V^T P^T with 32x32x16 MFMA, P in registers as above.
// One barrier a tile, between the halves of a stage:
//   stage j:  P_j = 2^(S_j - m) (VALU) between the MFMAs of S_{j+1}; the copies of K_{j+2} and V_j have landed; barrier;
//             the MFMAs of O with, between them, the requests for K_{j+3} and V_{j+1} and the row maxima of S_{j+1}
// Two workgroups on a CU hide each other's barriers.
constexpr int kTileRows = 128, kTileKeys = 64;

template <int D, bool F16, bool PREFIX>
__global__ void __launch_bounds__(256, 2) paged_tile_kernel(const Launch a)
{
    typedef typename Elem<F16>::T el;
    typedef typename Elem<F16>::x8 el8;
    typedef SubBlock<D> SB;
    constexpr int KS = D / 16, DB = D / 32;              // MFMAs of a score half; 32-row blocks of O^T
    constexpr int NQK = 2 * KS, NPV = 4 * DB, EPM = 32 / NQK;
    constexpr int PD = 4;                                // operand reads run that many MFMAs ahead
    constexpr int SLOT = 4 * SB::BYTES;
    constexpr uint32_t K0 = 0, V0 = 2 * SLOT;
    __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * SLOT];

    const PagedParams &p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hk = blockIdx.x % p.hkv, w = blockIdx.x / p.hkv;
    const int rg = a.groups - 1 - w % a.groups, x = w / a.groups;      // later rows see more keys: first
    Range r;
    int qn = p.seqlen, k0, k1;
    if constexpr (PREFIX) {
        r.b = 0, r.part = x, r.parts = a.parts, r.first = 0, r.len = p.prefix;
        k0 = x * a.chunk;
        k1 = min(p.prefix, k0 + a.chunk);
    } else {
        if (!find_range<true>(a, x, r)) return;
        qn = __builtin_amdgcn_readfirstlane(queries_of(p, r.b));
        k0 = r.part * r.chunk;
        k1 = (int)min((int64_t)r.len, (int64_t)k0 + r.chunk);
    }
    const int row0 = rg * kTileRows;
    if (!PREFIX && row0 >= qn * p.group && a.direct && r.parts == 1) return;         // (no row to store)
    const int l32 = lane & 31, hh = lane >> 5;
    const Row mine = row_of<PREFIX>(a, row0 + wave * 32 + l32, r.b, hk);
    int sees = k1, all_see = k1;
    if (!PREFIX && p.causal) {
        sees = min(k1, r.len - qn + mine.i + 1);
        all_see = min(k1, r.len - qn + (row0 + wave * 32) / p.group + 1);             // (of this wave's rows)
        k1 = min(k1, r.len - qn + min(row0 + kTileRows - 1, a.rows - 1) / p.group + 1);
    }
    const int n_tiles = max(0, (k1 - k0 + kTileKeys - 1) / kTileKeys);

    const int32_t *table = PREFIX ? p.prefix_table : p.table + r.b * p.tsb;
    const int last_page = max(k1 - 1, 0) >> p.pages.page_log2, in_page = (1 << p.pages.page_log2) - 1;
    el8 q[KS];
    {
        const uint16_t *src = p.q + mine.b * p.qsb + mine.i * p.qsn + mine.h * p.qsh + hh * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const el8 *>(src + 16 * s);
    }
    uint32_t koff[SB::UNITS], voff[SB::UNITS];
    SB::offsets(koff, lane, p.pages.ksn);
    SB::offsets(voff, lane, p.pages.vsn);
    const uint32_t lds = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) unsigned char *)ring);
    const uint16_t *const kh = p.k_cache + hk * p.pages.ksh, *const vh = p.v_cache + hk * p.pages.vsh;

    // the pages of a tile's sub-blocks, and of this wave's
    struct Tile { int id[4], mine; };
    auto tile_of = [&](int t) {
        Tile y;
#pragma unroll
        for (int s = 0; s < 4; ++s) y.id[s] = page_id(table, k0 + t * kTileKeys + s * kSub, p.pages.page_log2, last_page);
        y.mine = page_id(table, k0 + t * kTileKeys + wave * kSub, p.pages.page_log2, last_page);
        return y;
    };
    auto in_cache = [&](int id) { return (unsigned)id < (unsigned)p.pages.n_pages; };
    struct Source { i32x4 rsrc; uint32_t dst; };
    auto source = [&](const uint16_t *base, int64_t sp, int64_t sn, int t, const Tile &y, uint32_t slot) {
        const int key = k0 + t * kTileKeys + wave * kSub;
        const int n = __builtin_amdgcn_readfirstlane(in_cache(y.mine) ? min(max(k1 - key, 0), kSub) : 0);
        const int64_t id = n > 0 ? y.mine : 0;
        return Source{SB::descriptor(base + id * sp + (key & in_page) * sn, n, sn), (uint32_t)__builtin_amdgcn_readfirstlane(lds + slot + wave * SB::BYTES)};
    };
    auto k_source = [&](int t, const Tile &y, uint32_t slot) { return source(kh, p.pages.ksp, p.pages.ksn, t, y, K0 + slot); };
    auto v_source = [&](int t, const Tile &y, uint32_t slot) { return source(vh, p.pages.vsp, p.pages.vsn, t, y, V0 + slot); };

    // operand addresses.  K: row 32 kb + l32, elements 16 s + 8 hh .. + 7.  V: keys 16 u + 4 hh + 8 half + (L >> 2), 4 elements
    // from G16 * g16 + X * x + 4 (L & 3) on, transposed within 16 lanes: operand row 16 g16 + L of block x is that element of O
    constexpr int G16 = D == 128 ? 64 : 16, X = D == 128 ? 16 : 32;
    const int L = lane & 15, g16 = (lane >> 4) & 1;
    uint32_t ka[KS], va[DB][2];
#pragma unroll
    for (int s = 0; s < KS; ++s) ka[s] = lds + (l32 >> 4) * SB::BYTES + (l32 & 15) * (D * 2) + (((2 * s + hh) ^ swizzle<D>(l32 & 15)) * 16);
#pragma unroll
    for (int y = 0; y < DB; ++y)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = 4 * hh + 8 * half + (L >> 2), chunk = (G16 * g16 + X * y) / 8 + ((L >> 1) & 1);
            va[y][half] = lds + row * (D * 2) + ((chunk ^ swizzle<D>(row)) * 16) + (L & 1) * 8;
        }
    auto k_operand = [&](int n, uint32_t slot) {         // MFMA n: k-step n / 2, keys 32 (n % 2) ..
        return *LDS_PTR(const el8, ka[n >> 1] + K0 + slot + (n & 1) * 2 * SB::BYTES);
    };
    auto v_operand = [&](int n, uint32_t slot) {         // MFMA n: sub-block n / DB, block n % DB
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, va[n % DB][0] + V0 + slot + n / DB * SB::BYTES));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, va[n % DB][1] + V0 + slot + n / DB * SB::BYTES));
        return __builtin_bit_cast(el8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    f32x16 o[DB];
#pragma unroll
    for (int y = 0; y < DB; ++y)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[y][e] = 0.f;
    float m = kNone, l = 0.f, alpha = 1.f;
    uint64_t grown = 0;                                  // lanes whose row's maximum has grown with the next tile

    struct Scores { f32x16 s[2]; };
    auto masked = [&](Scores &z, int t, const Tile &y) {
        const int key = k0 + t * kTileKeys;
        bool there[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) there[s] = in_cache(y.id[s]);
        if (there[0] & there[1] & there[2] & there[3] & (key + kTileKeys <= all_see)) return;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int y = 32 * kb + 8 * (e >> 2) + 4 * hh + (e & 3);
                z.s[kb][e] = there[2 * kb + (e >> 3)] & (key + y < sees) ? z.s[kb][e] : -INFINITY;
            }
    };
    auto new_max = [&](float mx) {                       // of the raw scores, in both lanes of the row
        const float y = fmaxf(m, mx * p.scale_log2);
        grown = __builtin_amdgcn_ballot_w64(y > m);
        alpha = __builtin_amdgcn_exp2f(m - y);
        l *= alpha;
        m = y;
    };
    auto prob = [&](const Scores &z, int n) { return __builtin_amdgcn_exp2f(fmaf(z.s[n >> 4][n & 15], p.scale_log2, -m)); };

    el8 kpre[PD];
    Tile t1, t2, t3;                                     // pages of tiles j + 1, j + 2, j + 3
    // Stage j on the slots of its parity: cur -> P, next <- scores of tile j + 1, if there is one.
    auto stage = [&](auto parity, auto last, Scores &cur, Scores &next, int j) {
        constexpr uint32_t S0 = decltype(parity)::value * SLOT, S1 = SLOT - S0;      // slots of tile j and j + 1
        constexpr bool LAST = decltype(last)::value;
        el8 pr[4];
        float ex[EPM], sum[2] = {0.f, 0.f};
        auto pack = [&](int n) {
#pragma unroll
            for (int t = 0; t < EPM; ++t) pr[(n * EPM + t) >> 3][(n * EPM + t) & 7] = (el)ex[t];
        };
        if constexpr (!LAST) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) next.s[kb][e] = 0.f;
        }
        el8 ops[NQK + PD];
#pragma unroll
        for (int n = 0; n < PD; ++n) ops[n] = kpre[n];
#pragma unroll
        for (int n = 0; n < NQK; ++n) {
            if constexpr (!LAST) {
                if (n + PD < NQK) ops[n + PD] = k_operand(n + PD, S1);
                next.s[n & 1] = mfma16(ops[n], q[n >> 1], next.s[n & 1]);
            }
            float nx[EPM];
#pragma unroll
            for (int t = 0; t < EPM; ++t) nx[t] = prob(cur, n * EPM + t);
            if (n > 0) pack(n - 1);
#pragma unroll
            for (int t = 0; t < EPM; ++t) {
                ex[t] = nx[t];
                sum[t & 1] += nx[t];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        pack(NQK - 1);
        l += sum[0] + sum[1];
        Tile t4;
        if constexpr (!LAST) {
            masked(next, j + 1, t1);
            t4 = tile_of(j + 4);
        }
        wait_vmcnt<0>();
        wg_barrier();
        __builtin_amdgcn_sched_barrier(0);
        el8 vo[NPV + PD];
#pragma unroll
        for (int n = 0; n < PD; ++n) vo[n] = v_operand(n, S0);
        __builtin_amdgcn_sched_barrier(0);
        if (grown) {
#pragma unroll
            for (int y = 0; y < DB; ++y)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[y][e] *= alpha;
        }
        Source ks, vs;
        if constexpr (!LAST) {
            ks = k_source(j + 3, t3, S1);
            vs = v_source(j + 1, t1, S1);
            t1 = t2;
            t2 = t3;
            t3 = t4;
        }
        float mx = -INFINITY;
        static_for<NPV>([&](auto nc) {
            constexpr int n = decltype(nc)::value;
            if constexpr (n + PD < NPV) vo[n + PD] = v_operand(n + PD, S0);
            o[n % DB] = mfma16(vo[n], pr[n / DB], o[n % DB]);
            if constexpr (!LAST) {
                constexpr int PER = 2 * SB::UNITS / (NPV / 2);         // requests behind the first half of the MFMAs
                if constexpr (n < NPV / 2)
                    static_range<n * PER, (n + 1) * PER>([&](auto cc) {
                        constexpr int c = decltype(cc)::value, u = c % SB::UNITS;
                        if constexpr (c < SB::UNITS) SB::template unit<u>(vs.rsrc, voff[u], vs.dst);
                        else SB::template unit<u>(ks.rsrc, koff[u], ks.dst);
                    });
                constexpr int QUARTER = 32 / (NPV / 4);                // scores of a slot of the second quarter on
                if constexpr (n >= NPV / 4 && n < NPV / 2)
#pragma unroll
                    for (int e = (n - NPV / 4) * QUARTER; e < (n - NPV / 4 + 1) * QUARTER; ++e) mx = fmaxf(mx, next.s[e >> 4][e & 15]);
                if constexpr (n == NPV / 2) mx = pair_max(mx);
                if constexpr (n == NPV / 2 + 1) new_max(mx);
                if constexpr (n == NPV - 2)
#pragma unroll
                    for (int y = 0; y < PD; ++y) kpre[y] = k_operand(y, S0);          // of tile j + 2
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    if (n_tiles > 0) {
        const Tile t0 = tile_of(0);
        t1 = tile_of(1);
        t2 = tile_of(2);
        t3 = tile_of(3);
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[s]));      // (the queries before the copies: their wait would wait for both)
        auto whole = [&](const Source &s, const uint32_t (&off)[SB::UNITS]) {
            static_for<SB::UNITS>([&](auto u) { SB::template unit<decltype(u)::value>(s.rsrc, off[decltype(u)::value], s.dst); });
        };
        whole(k_source(0, t0, 0), koff);
        whole(k_source(1, t1, SLOT), koff);
        whole(v_source(0, t0, 0), voff);
        wait_vmcnt<2 * SB::UNITS>();
        wg_barrier();
        Scores even, odd;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) even.s[kb][e] = 0.f;
#pragma unroll
        for (int n = 0; n < NQK; ++n) even.s[n & 1] = mfma16(k_operand(n, 0), q[n >> 1], even.s[n & 1]);
        masked(even, 0, t0);
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 32; ++e) mx = fmaxf(mx, even.s[e >> 4][e & 15]);
        new_max(pair_max(mx));
        grown = 0;                                       // (the accumulators are zero)
        wait_vmcnt<0>();
        wg_barrier();
        whole(k_source(2, t2, 0), koff);
#pragma unroll
        for (int y = 0; y < PD; ++y) kpre[y] = k_operand(y, SLOT);
        // (two stages to a turn, so that the slots are constants; the last of an even number looks ahead to a tile of nothing)
        for (int j = 0; j + 1 < n_tiles; j += 2) {
            stage(std::integral_constant<int, 0>{}, std::false_type{}, even, odd, j);
            stage(std::integral_constant<int, 1>{}, std::false_type{}, odd, even, j + 1);
        }
        if (n_tiles & 1) stage(std::integral_constant<int, 0>{}, std::true_type{}, even, odd, n_tiles - 1);
    }

    // ---- results, through the LDS so that rows are written in whole lines ---------------------------------------
    wg_barrier();
    l += __shfl_xor(l, 32);
    const bool direct = !PREFIX && a.direct && r.parts == 1;
    const float f = !direct ? 1.f : l > 0.f ? 1.f / l : 0.f;
    constexpr int CH = D / 4;                            // 16-byte chunks of a row of 32-bit results
    float *const ro = reinterpret_cast<float *>(ring) + wave * 32 * D;
#pragma unroll
    for (int y = 0; y < DB; ++y)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int d = D == 128 ? 16 * y + 64 * (c >> 1) + 8 * (c & 1) + 4 * hh : 32 * y + 8 * c + 4 * hh;
            *reinterpret_cast<f32x4 *>(ro + l32 * D + (((d >> 2) ^ (l32 % CH)) << 2)) =
                f32x4{o[y][4 * c] * f, o[y][4 * c + 1] * f, o[y][4 * c + 2] * f, o[y][4 * c + 3] * f};
        }
    if (hh == 0) {
        const int row = row0 + wave * 32 + l32;
        if (direct) {
            if (p.lse && mine.stored && mine.i < qn)
                p.lse[((int64_t)mine.b * p.seqlen + mine.i) * p.hq + mine.h] = l > 0.f ? 0.6931471805599453f * (m + __builtin_amdgcn_logf(l)) : -INFINITY;
        } else if (mine.stored)
            (PREFIX ? a.prefix_ml : a.own_ml)[((int64_t)(PREFIX ? x : r.first + r.part) * p.hkv + hk) * a.rows + row] = make_float2(m, l);
    }
    constexpr int AT_ONCE = 64 / CH;                     // rows
    for (int y = lane / CH; y < 32; y += AT_ONCE) {
        const int row = row0 + wave * 32 + y, c = lane % CH;
        const Row z = row_of<PREFIX>(a, row, r.b, hk);
        const f32x4 v = *reinterpret_cast<const f32x4 *>(ro + y * D + ((c ^ (y % CH)) << 2));
        if (!z.stored) continue;
        if (direct) {
            if (z.i >= qn) continue;
            typedef el el4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<el4 *>(p.out + z.b * p.osb + z.i * p.osn + z.h * p.osh + 4 * c) = el4{(el)v[0], (el)v[1], (el)v[2], (el)v[3]};
        } else {
            float *dst = (PREFIX ? a.prefix_o : a.own_o) + (((int64_t)(PREFIX ? x : r.first + r.part) * p.hkv + hk) * a.rows + row) * D;
            *reinterpret_cast<f32x4 *>(dst + 4 * c) = v;
        }
    }
}

// ---- ranges joined --------------------------------------------------------------------------------------
// A workgroup is one row of one query head: its waves take the ranges in turn, a lane D / 64 elements.
template <int D, bool F16>
__global__ void __launch_bounds__(256) paged_join_kernel(const Launch a, const int prefix_rows, const int own_rows)
{
    typedef typename Elem<F16>::T el;
    constexpr int E = D / 64;
    typedef float fx __attribute__((ext_vector_type(E)));
    typedef el elx __attribute__((ext_vector_type(E)));
    __shared__ float red[4][D + 2];
    const PagedParams &p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x % p.hq, t = blockIdx.x / p.hq, i = t % p.seqlen, b = t / p.seqlen;
    if (i >= __builtin_amdgcn_readfirstlane(queries_of(p, b))) return;
    Range r;
    find_range<false>(a, b, r);
    if (a.direct && r.parts == 1) return;                // written already
    const int hk = h / p.group, g = h - hk * p.group;
    const int64_t own_row = (int64_t)i * p.group + g, prefix_row = ((int64_t)b * p.seqlen + i) * p.group + g;
    const int n = a.parts + r.parts;
    float m = kNone, l = 0.f;
    fx o;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int y = wave; y < n; y += 4) {
        const bool pre = y < a.parts;
        const int64_t slot = pre ? ((int64_t)y * p.hkv + hk) * prefix_rows + prefix_row : ((int64_t)(r.first + y - a.parts) * p.hkv + hk) * own_rows + own_row;
        const float2 ml = (pre ? a.prefix_ml : a.own_ml)[slot];
        const fx v = *reinterpret_cast<const fx *>((pre ? a.prefix_o : a.own_o) + slot * D + lane * E);
        const float mm = fmaxf(m, ml.x), f = __builtin_amdgcn_exp2f(m - mm), f2 = __builtin_amdgcn_exp2f(ml.x - mm);
        l = l * f + ml.y * f2;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + v[e] * f2;
        m = mm;
    }
    red[wave][D] = m;
    red[wave][D + 1] = l;
#pragma unroll
    for (int e = 0; e < E; ++e) red[wave][lane * E + e] = o[e];
    __syncthreads();
    if (wave != 0) return;
    for (int y = 1; y < 4; ++y) {
        const float my = red[y][D], mm = fmaxf(m, my), f = __builtin_amdgcn_exp2f(m - mm), f2 = __builtin_amdgcn_exp2f(my - mm);
        l = l * f + red[y][D + 1] * f2;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + red[y][lane * E + e] * f2;
        m = mm;
    }
    const float f = l > 0.f ? 1.f / l : 0.f;
    elx z;
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = (el)(o[e] * f);
    *reinterpret_cast<elx *>(p.out + b * p.osb + i * p.osn + h * p.osh + lane * E) = z;
    if (p.lse && lane == 0) p.lse[((int64_t)b * p.seqlen + i) * p.hq + h] = l > 0.f ? 0.6931471805599453f * (m + __builtin_amdgcn_logf(l)) : -INFINITY;
}

// ---- launch -----------------------------------------------------------------------------------------------
constexpr int kWaves = 4;
constexpr int kPlaces = 256;         // workgroups of the streaming kernel that the chip holds; twice as many of the other
constexpr int kFewRows = 64;         // up to that many rows of a unit are streamed

static int64_t up256(int64_t x) { return (x + 255) & ~(int64_t)255; }

struct Plan {
    Launch own, prefix;
    int64_t bytes;                   // of workspace
};

static Plan plan_of(const PagedParams &p, int head_dim)
{
    Plan y;
    Launch a = {};
    a.p = p;
    a.rows = p.seqlen * p.group;
    a.groups = a.rows <= kFewRows ? 1 : (a.rows + kTileRows - 1) / kTileRows;
    const int64_t items = (int64_t)p.batch * p.hkv * a.groups;
    const int places = a.rows <= kFewRows ? 4 * kPlaces : 2 * kPlaces;
    a.extra = p.max_len <= 256 || items >= places ? 0 : (int)std::max<int64_t>(1, places / (p.hkv * a.groups));
    a.direct = p.prefix == 0;
    y.own = a;
    y.bytes = 0;
    if (a.extra || !a.direct) {
        const int64_t rows = (int64_t)(p.batch + a.extra) * p.hkv * a.rows;
        y.bytes += up256(rows * head_dim * 4) + up256(rows * 8);
    }
    if (p.prefix) {
        Launch &z = y.prefix;
        z = a;
        z.rows = p.batch * a.rows;
        z.groups = z.rows <= kFewRows ? 1 : (z.rows + kTileRows - 1) / kTileRows;
        const int want = (int)std::max<int64_t>(1, (z.rows <= kFewRows ? 4 : 2) * kPlaces / ((int64_t)p.hkv * z.groups));
        z.chunk = std::max(128, (int)(((int64_t)p.prefix + want - 1) / want + 127) / 128 * 128);
        z.parts = (p.prefix + z.chunk - 1) / z.chunk;
        y.own.parts = z.parts;
        const int64_t rows = (int64_t)z.parts * p.hkv * z.rows;
        y.bytes += up256(rows * head_dim * 4) + up256(rows * 8);
    }
    unsigned char *at = p.workspace;
    if (a.extra || !a.direct) {
        const int64_t rows = (int64_t)(p.batch + a.extra) * p.hkv * a.rows;
        y.own.own_o = reinterpret_cast<float *>(at);
        y.own.own_ml = reinterpret_cast<float2 *>(at + up256(rows * head_dim * 4));
        at += up256(rows * head_dim * 4) + up256(rows * 8);
    }
    if (p.prefix) {
        const int64_t rows = (int64_t)y.prefix.parts * p.hkv * y.prefix.rows;
        y.own.prefix_o = y.prefix.prefix_o = reinterpret_cast<float *>(at);
        y.own.prefix_ml = y.prefix.prefix_ml = reinterpret_cast<float2 *>(at + up256(rows * head_dim * 4));
    }
    return y;
}

size_t paged_workspace_bytes(const PagedParams &p, int head_dim) { return (size_t)plan_of(p, head_dim).bytes; }

template <int D, bool F16, bool PREFIX> static void attend(const Launch &a, int64_t ranges, hipStream_t stream)
{
    const unsigned grid = (unsigned)(ranges * a.p.hkv * a.groups);
    if (a.rows <= 16) paged_stream_kernel<D, kWaves, 1, F16, PREFIX><<<grid, kWaves * 64, 0, stream>>>(a);
    else if (a.rows <= 32) paged_stream_kernel<D, kWaves, 2, F16, PREFIX><<<grid, kWaves * 64, 0, stream>>>(a);
    else if (a.rows <= kFewRows) paged_stream_kernel<D, kWaves, 4, F16, PREFIX><<<grid, kWaves * 64, 0, stream>>>(a);
    else paged_tile_kernel<D, F16, PREFIX><<<grid, 256, 0, stream>>>(a);
}

template <int D, bool F16> static hipError_t launch(const PagedParams &p, hipStream_t stream)
{
    const Plan y = plan_of(p, D);
    if (p.prefix) attend<D, F16, true>(y.prefix, y.prefix.parts, stream);
    attend<D, F16, false>(y.own, p.batch + y.own.extra, stream);
    if (y.own.extra || !y.own.direct)
        paged_join_kernel<D, F16><<<(unsigned)(p.batch * p.seqlen * p.hq), 256, 0, stream>>>(y.own, p.batch * y.own.rows, y.own.rows);
    return hipGetLastError();
}

hipError_t launch_paged(const PagedParams &p, int head_dim, bool f16, hipStream_t stream)
{
    if (head_dim == 128) return f16 ? launch<128, true>(p, stream) : launch<128, false>(p, stream);
    if (head_dim == 64) return f16 ? launch<64, true>(p, stream) : launch<64, false>(p, stream);
    return hipErrorInvalidValue;
}

}  // namespace bsfa
