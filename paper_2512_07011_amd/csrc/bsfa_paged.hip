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
    // requests the sub-block whose first row is at `src`; of its rows only `n` exist, the others become 0
    __device__ __forceinline__ static void copy(const uint16_t *src, int n, int64_t stride, const uint32_t (&off)[UNITS], uint32_t lds)
    {
        const uint64_t at = reinterpret_cast<uint64_t>(src);
        const i32x4 rsrc = {(int)(uint32_t)at, (int)((uint32_t)(at >> 32) & 0xffffu), n > 0 ? ((n - 1) * (int)stride + D) * 2 : 0, 0x00020000};
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds);
        asm volatile("s_nop 3" : : "s"(rsrc));           // (a descriptor from a vector instruction is read 5 states later at the earliest)
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %3, 0 offen lds"
                         : : "v"(off[u]), "s"(dst), "n"(u * kUnit), "s"(rsrc) : "memory", "m0", "scc");
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
    auto exist = [&](int key, int id) { return (unsigned)id < (unsigned)p.pages.n_pages ? min(max(k1 - key, 0), kSub) : 0; };
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
constexpr int kPlaces = 256;         // workgroups that the chip holds

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
    a.groups = (a.rows + 63) / 64;
    const int64_t items = (int64_t)p.batch * p.hkv * a.groups;
    a.extra = p.max_len <= 256 || items >= 4 * kPlaces ? 0 : (int)std::max<int64_t>(1, (4 * kPlaces) / (p.hkv * a.groups));
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
        z.groups = (z.rows + 63) / 64;
        const int want = (int)std::max<int64_t>(1, 4 * kPlaces / ((int64_t)p.hkv * z.groups));
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

template <int D, bool F16, bool PREFIX> static void stream_keys(const Launch &a, int64_t ranges, hipStream_t stream)
{
    const unsigned grid = (unsigned)(ranges * a.p.hkv * a.groups);
    if (a.rows <= 16) paged_stream_kernel<D, kWaves, 1, F16, PREFIX><<<grid, kWaves * 64, 0, stream>>>(a);
    else if (a.rows <= 32) paged_stream_kernel<D, kWaves, 2, F16, PREFIX><<<grid, kWaves * 64, 0, stream>>>(a);
    else paged_stream_kernel<D, kWaves, 4, F16, PREFIX><<<grid, kWaves * 64, 0, stream>>>(a);
}

template <int D, bool F16> static hipError_t launch(const PagedParams &p, hipStream_t stream)
{
    const Plan y = plan_of(p, D);
    if (p.prefix) stream_keys<D, F16, true>(y.prefix, y.prefix.parts, stream);
    stream_keys<D, F16, false>(y.own, p.batch + y.own.extra, stream);
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
