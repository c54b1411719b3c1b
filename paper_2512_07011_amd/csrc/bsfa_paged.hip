// Attention of new tokens over a paged K/V cache for gfx950, wave64, bf16 or fp16 MFMA:
//     o_i = sum_t softmax_t(q_i k_t / sqrt(d)) v_t
// over the tokens t that query i sees: those its sequence has in its own pages (causal: up to i's own place) and those of a
// prefix that all sequences share.  One pass over the keys with a running maximum m (fp16: 7 less, kLift), normaliser l and unscaled accumulator
// O; ranges of keys are worked on apart and joined by
//     m = max m_x,  l = sum l_x 2^(m_x - m),  O = sum O_x 2^(m_x - m)          (log2 units).
// The (query token, query head) pairs that read one KV head are the rows of a unit: one sequence's, or for the prefix
// everybody's.
//
// What bounds it.  Few rows to a key (decoding: the query heads of a KV head, 512 bytes of K and V for 4 d times as many
// operations): memory.  64 sequences of 1K to 8K tokens, 905 MB: 163 us, 5.6 TB/s; two of 128K, 1.07 GB: 185 us, 5.8 TB/s (a
// large copy moves 4.9 TB/s on the same card, read and written bytes together).  Many rows (a chunk of a prompt, a batch behind one
// prefix): the matrix pipe and the exponentials beside it.  2048 tokens behind 30K of 32 heads: 965 us, 1.11 PFLOP/s (other cards
// 925 to 1000 us), the pipe busy in 67 % of the cycles at 1.56 GHz (a large library product reaches 1.32 PFLOP/s).  Small calls: their chain of dependent trips to memory --
// lengths, page, keys, the ranges' results -- 9 us for a thousand tokens.
#include "bsfa_dev.h"

#include <algorithm>

namespace bsfa {

typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 mfma32(bf16x8_t a, bf16x8_t b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma32(f16x8_t a, f16x8_t b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x4 mfma16x16(s16x4 a, Elem<false>::x4 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, __builtin_bit_cast(s16x4, b), c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16x16(s16x4 a, Elem<true>::x4 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(Elem<true>::x4, a), b, c, 0, 0, 0); }

constexpr float kNone = -3.0e38f;    // running maximum of a row that has seen no key: finite, below any score
// A row's running maximum follows its scores only when they have outgrown it by more than this (log2 units): weights stay
// below 2^8, which costs no precision, and accumulators are hardly ever rescaled (with a growth of nothing allowed, some row of
// 32 grows in one tile of five over 32K keys).
constexpr float kSlack = 8.f;
// fp16: what a row's exponent m is kept below its maximum by, so that weights reach 2^15 at most (with kSlack) and only those below
// 2^-32 of the largest round to 0.  Without it that was 2^-25, and 16384 keys of e^-17.5 of one other's weight each were lost,
// of e^-16 came out 6 % off.  bf16 has the exponents of 32 bits.  l and the accumulators have the same factor, and (m, l) mean
// the same wherever ranges are joined.
template <bool F16> constexpr float kLift = F16 ? 7.f : 0.f;
constexpr int kSub = 16;             // keys that lie in one page whatever its size

struct Launch {
    PagedParams p;
    // The sequences' own tokens: a unit of `rows` rows each, `groups` workgroups side by side.  shares > 0: the batch's tokens
    // are dealt to so many workgroups evenly (even_share), min_share sub-blocks or more each; 0: one to a sequence.
    int rows, groups, shares, min_share, near, range_cost;
    // The prefix: one unit of prefix_rows rows, ranges of prefix_chunk keys.
    int prefix_rows, prefix_groups, prefix_parts, prefix_chunk;
    // Unscaled results of ranges [slot][hkv][rows][d] and their (m, l); slots: see Range, and the prefix's ranges.
    float *own_o, *prefix_o;
    float2 *own_ml, *prefix_ml;
    int2 *own_ranges;                // shares > 0: first slot and number of ranges of every sequence
    int own_slots;
    bool direct;                     // a sequence in one range is written to out at once
};

// The kernels' arguments as they lie in constant memory, asked for anew: each part of a kernel reads what it needs when it
// begins, and what only the end of a range needs takes no scalar registers during its loop.
typedef const __attribute__((address_space(4))) Launch Args;
typedef const __attribute__((address_space(4))) PagedParams Params;
__device__ __forceinline__ Args &arguments()
{
    uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(Args *)at;
}
// The same number, computed anew by whatever depends on it.
__device__ __forceinline__ int anew(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// ---- ranges of keys -------------------------------------------------------------------------------------
struct Range {
    int b, len, new_tokens;          // sequence, its tokens, its rows' tokens
    int k0, k1;                      // keys
    int slot;                        // where the result goes ...
    bool whole;                      // ... unless this is all of the sequence
};

__device__ __forceinline__ int queries_of(Params &p, int b) { return p.q_lens ? min(max(p.q_lens[b], 0), p.seqlen) : p.seqlen; }
// A sequence's tokens and its rows' tokens.  One that rests, with tokens but none to compute, counts as one without: nobody sees them.
__device__ __forceinline__ void lengths_of(Params &p, int b, int &len, int &news)
{
    const int n = p.cache_lens[b];
    news = queries_of(p, b);
    len = news ? min(max(n, 0), p.max_len) : 0;
}
// What a sequence counts as, in sub-blocks: its own and what a range's beginning and end take, at least a workgroup's share
__device__ __forceinline__ int units_of(Args &a, int len) { return max((int)((unsigned)(len + kSub - 1) / kSub) + a.range_cost, a.min_share); }

// The batch's sub-blocks in a row, dealt to `shares` workgroups evenly: workgroup x has those from x * share on, which may
// begin and end inside sequences.  A border between two workgroups that lies no more than `near` sub-blocks from a border
// between two sequences is moved there: a range more costs more than that.  A workgroup or a sequence begins with every
// range, so the range of workgroup x in sequence b has slot x + b.  The shares follow from the lengths on the device: a
// captured launch stays even as sequences grow.
struct Share {
    int share, near;                 // sub-blocks of a workgroup; see above
    int b, before, len, new_tokens;  // a sequence, the sub-blocks before it, its tokens, its rows' tokens
    int b0, lens, news;              // of sequence b0 + lane
};
__device__ __forceinline__ void load_lengths(Params &p, int b0, int &lens, int &news)
{
    lengths_of(p, min(b0 + (int)(threadIdx.x & 63), p.batch - 1), lens, news);
}
__device__ __forceinline__ void take_sequence(Params &p, int b, Share &y)
{
    if (b >= y.b0 + 64) load_lengths(p, y.b0 = b, y.lens, y.news);
    y.b = b;
    y.len = __builtin_amdgcn_readlane(y.lens, b - y.b0);
    y.new_tokens = __builtin_amdgcn_readlane(y.news, b - y.b0);
}
// sum over lanes 0 .. l: inside rows of 16 lanes, then each row's last lane to the rows behind it
__device__ __forceinline__ int scan_lanes(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);       // row_shr:2
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);       // row_shr:4
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);       // row_shr:8
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // row_bcast:31 into rows 2 and 3
    return x;
}
// The sequence that holds sub-block x * share; every wave for itself.  False: there is none.
__device__ __forceinline__ bool even_share(Args &a, int x, Share &y)
{
    Params &p = a.p;
    const int lane = threadIdx.x & 63;
    // sub-blocks of sequences b0 .. b0 + lane; all 64 of them
    auto scan = [&](int b0, int lens) { return scan_lanes(b0 + lane < p.batch ? units_of(a, lens) : 0); };
    auto last = [](int upto) { return __builtin_amdgcn_readlane(upto, 63); };
    y.b0 = 0;
    load_lengths(p, 0, y.lens, y.news);
    int upto = scan(0, y.lens), total = last(upto);
    for (int b0 = 64; b0 < p.batch; b0 += 64) {
        int lens, news;
        load_lengths(p, b0, lens, news);
        total += last(scan(b0, lens));
    }
    y.share = max((total + a.shares - 1) / a.shares, a.min_share);
    y.near = max(min(a.near, y.share / 4), a.range_cost);
    int before = 0;
    while (true) {
        const int sum = last(upto);
        if ((int64_t)x * y.share < before + sum) {
            const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + upto > x * y.share));
            take_sequence(p, y.b0 + l, y);
            y.before = before + __builtin_amdgcn_readlane(upto, l) - units_of(a, y.len);
            return true;
        }
        before += sum;
        if (y.b0 + 64 >= p.batch) return false;
        load_lengths(p, y.b0 += 64, y.lens, y.news);
        upto = scan(y.b0, y.lens);
    }
}

// The sequences' own tokens that are workgroup x's: f for every range.  (KEEP: the lengths that are at hand stay in two
// vector registers in the meantime, and the next range does not wait for its own.)
template <bool KEEP, class F> __device__ __forceinline__ void own_ranges(int hk, int x, int rg, F &&f)
{
    Share y;
    int from = 0, to = 0x7fffffff;                       // (all of one sequence)
    {
        Args &a = arguments();
        if (a.shares) {
            if (!even_share(a, x, y)) return;
            from = x * y.share;
            to = from + y.share;
        } else {
            y.b = x;
            y.before = y.b0 = 0;
            lengths_of(a.p, x, y.len, y.new_tokens);
            y.len = __builtin_amdgcn_readfirstlane(y.len);
            y.new_tokens = __builtin_amdgcn_readfirstlane(y.new_tokens);
        }
    }
    while (true) {
        Args &a = arguments();
        Range r;
        const int end = y.before + units_of(a, y.len);
        // borders moved to this sequence's: where it begins or ends close to them
        int lo = from, hi = to;
        if (a.shares) {
            if (lo > y.before) lo = lo - y.before <= y.near ? y.before : end - lo <= y.near ? end : lo;
            if (hi < end) hi = hi - y.before <= y.near ? y.before : end - hi <= y.near ? end : hi;
        }
        if (hi <= y.before) return;                      // (the next workgroup's)
        r.b = y.b;
        r.len = y.len;
        r.new_tokens = y.new_tokens;
        r.k0 = max(lo - y.before, 0) * kSub;
        r.k1 = end <= hi ? r.len : min((hi - y.before) * kSub, r.len);
        r.slot = a.shares ? x + y.b : x;
        r.whole = lo <= y.before && end <= hi;
        // where the join finds the sequence's ranges: the borders behind this one that lie inside it begin one each
        if (a.shares && lo <= y.before && hk == 0 && rg == 0 && threadIdx.x == 0)
            a.own_ranges[y.b] = make_int2(r.slot, max((end - y.near - 1) / y.share - x, 0) + 1);
        if (lo < end) {                                  // (else the workgroup before has all of it)
            f(r);
            __syncthreads();                             // (the LDS is free again)
        }
        Args &z = arguments();
        y.before = end;
        if (!z.shares || end >= to || y.b + 1 >= z.p.batch) return;
        if constexpr (KEEP) take_sequence(z.p, y.b + 1, y);
        else {
            lengths_of(z.p, ++y.b, y.len, y.new_tokens);
            y.len = __builtin_amdgcn_readfirstlane(y.len);
            y.new_tokens = __builtin_amdgcn_readfirstlane(y.new_tokens);
        }
    }
}

__device__ __forceinline__ Range prefix_range(Args &a, int x)
{
    Range r;
    r.b = 0;
    r.len = a.p.prefix;
    r.new_tokens = a.p.seqlen;
    r.k0 = x * a.prefix_chunk;
    r.k1 = min(r.k0 + a.prefix_chunk, r.len);
    r.slot = x;
    r.whole = false;
    return r;
}

// ---- tiles of keys in LDS ---------------------------------------------------------------------------
// Kept as sub-blocks of 16 keys, rows of 2 D bytes, without gaps (a direct copy's LDS side is linear).  The 16-byte chunks
// of a row are permuted among themselves, c -> c ^ swizzle(row), on the global side of the copy, so that no two of the lanes
// that an LDS read serves together meet in a bank: 16 rows at one chunk (K, 16 bytes a lane); V, 32 lanes of 8 bytes: rows
// 0 .. 7 (and 8 .. 15) at a pair of chunks, or rows 0 .. 3 (4 .. 7, ...) at two pairs, 8 chunks apart (width 64: 2).
template <int D> __device__ __forceinline__ int swizzle(int row)
{
    return D == 128 ? (row << 1 & 14) | (row >> 3 & 1) : (row << 1 & 4) | (row >> 1 & 2) | (row >> 3 & 1);
}

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
template <bool PREFIX> __device__ __forceinline__ Row row_of(int rows, int group, int seqlen, int r, int b, int hk)
{
    const int rr = min(r, rows - 1), t = rr / group;
    Row x;
    x.b = PREFIX ? t / seqlen : b;
    x.i = PREFIX ? t - x.b * seqlen : t;
    x.h = hk * group + rr - t * group;
    x.stored = r < rows;
    return x;
}

// A row's result: the sum of its weights l and their maximum's exponent m give the log-sum-exp.  Only l = 0 is a row that sees
// nothing: a query that is not finite makes l NaN, and both have to show it.
__device__ __forceinline__ float natural_lse(float m, float l) { return l == 0.f ? -INFINITY : 0.6931471805599453f * (m + __builtin_amdgcn_logf(l)); }
__device__ __forceinline__ float normaliser(float l) { return l == 0.f ? 0.f : 1.f / l; }

// ---- few rows: keys streamed once ---------------------------------------------------------------------
// A workgroup is four waves on 16 * NRT rows of one unit and one range of keys.  Every wave takes tiles of 16 keys of its own
// (every fourth), with a ring of kStages tiles in LDS that only it reads: no barrier until the waves' results are joined at
// the end, and K and V go from memory to LDS without a register.  16 keys and two workgroups to a CU, or 32 keys and one, have
// the same bytes in flight, but two hide each other's beginnings and ends (256 sequences of 40 to 400 tokens 49 / 31 us, 128K tokens alike).
//   S^T = K Q^T     16x16x32 MFMA, fp32; column = row of the unit, so that a row's scores lie in four lanes
//   O^T += V^T P^T  16x16x16 MFMA, V^T through the transposing LDS read; the accumulator layout of S^T is the operand layout
//                   of P^T, so P never leaves the registers
// Rounded: P to the element type for the second product (its operands have it); l sums the unrounded fp32 values.
constexpr int kStages = 2;
constexpr int kWaves = 4;

template <int D, int NRT> struct StreamLds {
    static constexpr int STAGE = 2 * SubBlock<D>::BYTES;                 // K and V of a tile
    unsigned char ring[kWaves * kStages * STAGE];
    float m[kWaves][kSub * NRT], l[kWaves][kSub * NRT];                  // (where the waves' results are joined)
};

template <int D, int NRT, bool F16, bool PREFIX>
__device__ __forceinline__ void stream_range(Args &a, const Range r, int hk, int rg, StreamLds<D, NRT> &shared)
{
    typedef typename Elem<F16>::T el;
    typedef typename Elem<F16>::x8 el8;
    typedef typename Elem<F16>::x4 el4;
    typedef SubBlock<D> SB;
    constexpr int NW = kWaves;
    constexpr int KEYS = kSub;
    constexpr int KI = D / 32;                           // MFMAs of a score tile
    constexpr int DB = D / 16;                           // 16-row blocks of O^T
    constexpr int STAGE = StreamLds<D, NRT>::STAGE;
    constexpr int PER_STAGE = 2 * SB::UNITS;             // copies
    constexpr int OPITCH = D + 4;                        // floats of a row where the waves' results are joined
    static_assert(NW * kSub * OPITCH * 4 <= NW * kStages * STAGE, "joining fits the ring");

    Params &p = a.p;
    const bool masked = !PREFIX && p.causal;
    const int lane = anew(threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (anew: nothing of a lane's is kept from range to range)
    const int qn = r.new_tokens;
    const int k0 = r.k0, rows = PREFIX ? a.prefix_rows : a.rows;
    int k1 = r.k1;
    const int row0 = rg * kSub * NRT;
    if (!PREFIX && row0 >= qn * p.group) return;         // (no row that anybody reads)
    const int n16 = lane & 15, quad = lane >> 4;
    int sees[NRT];                                       // keys below it are visible to this lane's row
    int all_see = k1;                                    // ... to every row
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        sees[t] = k1;
        if (masked) sees[t] = min(k1, r.len - qn + row_of<PREFIX>(rows, p.group, p.seqlen, row0 + t * kSub + n16, r.b, hk).i + 1);
    }
    if (masked) {
        all_see = min(k1, r.len - qn + row0 / p.group + 1);
        k1 = min(k1, r.len - qn + min(row0 + kSub * NRT - 1, rows - 1) / p.group + 1);      // keys that some row sees
    }

    const int32_t *table = PREFIX ? p.prefix_table : p.table + r.b * p.tsb;
    const int last_page = max(k1 - 1, 0) >> p.pages.page_log2, in_page = (1 << p.pages.page_log2) - 1;
    el8 q[NRT][KI];
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        const Row y = row_of<PREFIX>(rows, p.group, p.seqlen, row0 + t * kSub + n16, r.b, hk);
        const uint16_t *src = p.q + y.b * p.qsb + y.i * p.qsn + y.h * p.qsh + quad * 8;
#pragma unroll
        for (int i = 0; i < KI; ++i) q[t][i] = *reinterpret_cast<const el8 *>(src + 32 * i);
    }
    uint32_t koff[SB::UNITS], voff[SB::UNITS];
    SB::offsets(koff, lane, p.pages.ksn);
    SB::offsets(voff, lane, p.pages.vsn);
    const uint32_t mine = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) unsigned char *)shared.ring) + wave * kStages * STAGE;
    const uint16_t *const kh = p.k_cache + hk * p.pages.ksh, *const vh = p.v_cache + hk * p.pages.vsh;

    // Pages: lane i holds the page of this wave's tile 64 w + i of window w, read once for 64 tiles (the wait for them is one
    // for the copies in flight, too).  Through the scalar cache a page would be in the way of every LDS read, whose waits
    // cannot tell the two apart.
    constexpr int STEP = KEYS * NW;
    const int first = k0 + KEYS * wave;
    int window = 0;
    auto page_of = [&](int tile) {
        if ((tile & 63) == 0) window = table[min((first + (tile + lane) * STEP) >> p.pages.page_log2, last_page)];
        return __builtin_amdgcn_readlane(window, tile & 63);
    };
    // keys of a tile that exist: none where it lies behind the range or its page is none of the cache's
    auto exist = [&](int key, int id) { return __builtin_amdgcn_readfirstlane((unsigned)id < (unsigned)p.pages.n_pages ? min(max(k1 - key, 0), kSub) : 0); };
    auto request = [&](int key, int page, int n, uint32_t at) {
        const int64_t id = n > 0 ? page : 0, place = key & in_page;
        SB::copy(kh + id * p.pages.ksp + place * p.pages.ksn, n, p.pages.ksn, koff, at);
        SB::copy(vh + id * p.pages.vsp + place * p.pages.vsn, n, p.pages.vsn, voff, at + SB::BYTES);
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
    for (int x = 0; x < DB; ++x) va[x] = vrow * (D * 2) + (((2 * x + ((n16 >> 1) & 1)) ^ swizzle<D>(vrow)) * 16) + (n16 & 1) * 8 + SB::BYTES;

    // the queries arrive before the copies are requested: a wait for them would wait for the copies, too
#pragma unroll
    for (int t = 0; t < NRT; ++t)
#pragma unroll
        for (int i = 0; i < KI; ++i) asm volatile("" : "+v"(q[t][i]));
    int now, next;                                       // keys of the tile at hand and of the next one that exist
    {
        const int page = page_of(0), page2 = page_of(1);
        now = exist(first, page);
        next = exist(first + STEP, page2);
        request(first, page, now, mine);
        request(first + STEP, page2, next, mine + STAGE);
    }
    uint32_t at = mine;
    for (int tile = 0, key = first; key < k1; ++tile, key += STEP) {
        wait_vmcnt<PER_STAGE>();
        asm volatile("" : : : "memory");
        f32x4 s[NRT];
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const el8 kk = *LDS_PTR(const el8, at + ka[i]);
#pragma unroll
            for (int t = 0; t < NRT; ++t) s[t] = mfma32(kk, q[t][i], i == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[t]);
        }
        if (now < KEYS || key + KEYS > all_see) {
#pragma unroll
            for (int t = 0; t < NRT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int y = 4 * quad + e;
                    if (!((y < now) & (key + y < sees[t]))) s[t][e] = -INFINITY;
                }
        }
        el4 pr[NRT];
#pragma unroll
        for (int t = 0; t < NRT; ++t) {
            float mx = quad_max(fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3]))) * p.scale_log2 - kLift<F16>;
            if (__builtin_amdgcn_ballot_w64(mx > m[t] + kSlack)) {
                mx = mx > m[t] + kSlack ? mx : m[t];
                const float f = __builtin_amdgcn_exp2f(m[t] - mx);
                l[t] *= f;
#pragma unroll
                for (int x = 0; x < DB; ++x) o[t][x] *= f;
                m[t] = mx;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = __builtin_amdgcn_exp2f(fmaf(s[t][e], p.scale_log2, -m[t]));
                l[t] += y;
                pr[t][e] = (el)y;
            }
        }
#pragma unroll
        for (int x = 0; x < DB; ++x) {
            const s16x4 vv = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, at + va[x]));
#pragma unroll
            for (int t = 0; t < NRT; ++t) o[t][x] = mfma16x16(vv, pr[t], o[t][x]);
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0): this tile has been read
        asm volatile("" : : : "memory");
        const int page = page_of(tile + 2), n = exist(key + 2 * STEP, page);
        request(key + 2 * STEP, page, n, at);
        now = next;
        next = n;
        at ^= mine ^ (mine + STAGE);
    }

    // ---- the waves' results joined, 16 rows at a time --------------------------------------------------
    wait_vmcnt<0>();
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        l[t] = quad_sum(l[t]);
        if (quad == 0) {
            shared.m[wave][t * kSub + n16] = m[t];
            shared.l[wave][t * kSub + n16] = l[t];
        }
    }
    float *const ro = reinterpret_cast<float *>(shared.ring);
    constexpr int TPR = NW * 64 / kSub, DPT = D / TPR;   // threads of a row, elements of a thread
    const int tid = anew(threadIdx.x), jr = tid / TPR, jd = tid % TPR * DPT;
    Args &z = arguments();
    const int end_rows = PREFIX ? z.prefix_rows : z.rows;
    const bool direct = z.direct && r.whole;
#pragma unroll
    for (int t = 0; t < NRT; ++t) {
        __syncthreads();
#pragma unroll
        for (int x = 0; x < DB; ++x) *reinterpret_cast<f32x4 *>(ro + (wave * kSub + n16) * OPITCH + 16 * x + 4 * quad) = o[t][x];
        __syncthreads();
        const int row = row0 + t * kSub + jr;
        float mm = kNone, ll = 0.f, oo[DPT];
#pragma unroll
        for (int v = 0; v < NW; ++v) mm = fmaxf(mm, shared.m[v][t * kSub + jr]);
#pragma unroll
        for (int d = 0; d < DPT; ++d) oo[d] = 0.f;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const float f = __builtin_amdgcn_exp2f(shared.m[v][t * kSub + jr] - mm);
            ll = fmaf(f, shared.l[v][t * kSub + jr], ll);
#pragma unroll
            for (int d = 0; d < DPT; ++d) oo[d] = fmaf(f, ro[(v * kSub + jr) * OPITCH + jd + d], oo[d]);
        }
        const Row y = row_of<PREFIX>(end_rows, z.p.group, z.p.seqlen, row, r.b, hk);
        if (!y.stored) continue;
        if (direct) {
            if (y.i >= qn) continue;
            const float f = normaliser(ll);
            uint16_t *dst = z.p.out + y.b * z.p.osb + y.i * z.p.osn + y.h * z.p.osh + jd;
            typedef el elx __attribute__((ext_vector_type(DPT)));
            elx w;
#pragma unroll
            for (int d = 0; d < DPT; ++d) w[d] = (el)(oo[d] * f);
            *reinterpret_cast<elx *>(dst) = w;
            if (z.p.lse && jd == 0) z.p.lse[((int64_t)y.b * z.p.seqlen + y.i) * z.p.hq + y.h] = natural_lse(mm, ll);
        } else {
            const int64_t at = ((int64_t)r.slot * z.p.hkv + hk) * end_rows + row;
            float *dst = (PREFIX ? z.prefix_o : z.own_o) + at * D + jd;
#pragma unroll
            for (int d = 0; d < DPT; d += 4) *reinterpret_cast<f32x4 *>(dst + d) = f32x4{oo[d], oo[d + 1], oo[d + 2], oo[d + 3]};
            if (jd == 0) (PREFIX ? z.prefix_ml : z.own_ml)[at] = make_float2(mm, ll);
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

template <int D> struct TileLds {
    unsigned char ring[16 * SubBlock<D>::BYTES];
};

template <int D, bool F16, bool PREFIX>
__device__ __forceinline__ void tile_range(Args &a, const Range r, int hk, int rg, TileLds<D> &shared)
{
    typedef typename Elem<F16>::T el;
    typedef typename Elem<F16>::x8 el8;
    typedef SubBlock<D> SB;
    constexpr int KS = D / 16, DB = D / 32;              // MFMAs of a score half; 32-row blocks of O^T
    constexpr int NQK = 2 * KS, NPV = 4 * DB, EPM = 32 / NQK;
    constexpr int PD = D == 64 ? 3 : 4;                  // operand reads run that many MFMAs ahead (64: three waves to a SIMD, 168 registers)
    constexpr int SLOT = 4 * SB::BYTES;
    constexpr uint32_t K0 = 0, V0 = 2 * SLOT;

    Params &p = a.p;
    const bool causal = !PREFIX && p.causal;
    const int lane = anew(threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (anew: nothing of a lane's is kept from range to range)
    const int qn = r.new_tokens;
    const int k0 = r.k0, rows = PREFIX ? a.prefix_rows : a.rows;
    int k1 = r.k1;
    const int row0 = rg * kTileRows;
    const bool direct = a.direct && r.whole;
    if (!PREFIX && row0 >= qn * p.group) return;         // (no row that anybody reads)
    const int l32 = lane & 31, hh = lane >> 5;
    const Row mine = row_of<PREFIX>(rows, p.group, p.seqlen, row0 + wave * 32 + l32, r.b, hk);
    int sees = k1, all_see = k1;
    if (causal) {
        sees = min(k1, r.len - qn + mine.i + 1);
        all_see = min(k1, r.len - qn + (row0 + wave * 32) / p.group + 1);             // (of this wave's rows)
        k1 = min(k1, r.len - qn + min(row0 + kTileRows - 1, rows - 1) / p.group + 1);
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
    const uint32_t lds = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) unsigned char *)shared.ring);
    const uint16_t *const kh = p.k_cache + hk * p.pages.ksh, *const vh = p.v_cache + hk * p.pages.vsh;

    // Pages of a tile's sub-blocks, one to a lane (of four).  They arrive with the copies that are requested next to them; through
    // the scalar cache they would be in the way of every LDS read, whose waits cannot tell the two apart.
    auto tile_of = [&](int t) { return table[min((k0 + t * kTileKeys + (lane & 3) * kSub) >> p.pages.page_log2, last_page)]; };
    // which of the four are pages of the cache
    auto in_cache = [&](int pages) { return (uint32_t)__builtin_amdgcn_ballot_w64((unsigned)pages < (unsigned)p.pages.n_pages) & 15u; };
    struct Source { i32x4 rsrc; uint32_t dst; };
    auto source = [&](const uint16_t *base, int64_t sp, int64_t sn, int t, int pages, uint32_t slot) {
        const int key = k0 + t * kTileKeys + wave * kSub, page = __builtin_amdgcn_readlane(pages, wave);
        const int n = __builtin_amdgcn_readfirstlane((unsigned)page < (unsigned)p.pages.n_pages ? min(max(k1 - key, 0), kSub) : 0);
        const int64_t id = n > 0 ? page : 0;
        return Source{SB::descriptor(base + id * sp + (key & in_page) * sn, n, sn), (uint32_t)__builtin_amdgcn_readfirstlane(lds + slot + wave * SB::BYTES)};
    };
    auto k_source = [&](int t, int pages, uint32_t slot) { return source(kh, p.pages.ksp, p.pages.ksn, t, pages, K0 + slot); };
    auto v_source = [&](int t, int pages, uint32_t slot) { return source(vh, p.pages.vsp, p.pages.vsn, t, pages, V0 + slot); };

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
    auto masked = [&](Scores &z, int t, int pages) {
        const int key = k0 + t * kTileKeys;
        const uint32_t there = in_cache(pages);
        if ((there == 15u) & (key + kTileKeys <= all_see)) return;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int y = 32 * kb + 8 * (e >> 2) + 4 * hh + (e & 3);
                if (!((there >> (2 * kb + (e >> 3)) & 1u) & (key + y < sees))) z.s[kb][e] = -INFINITY;
            }
    };
    auto new_max = [&](float mx) {                       // of the raw scores, in both lanes of the row
        mx = mx * p.scale_log2 - kLift<F16>;
        const float y = mx > m + kSlack ? mx : m;
        grown = __builtin_amdgcn_ballot_w64(y > m);
        alpha = __builtin_amdgcn_exp2f(m - y);
        l *= alpha;
        m = y;
    };
    auto prob = [&](const Scores &z, int n) { return __builtin_amdgcn_exp2f(fmaf(z.s[n >> 4][n & 15], p.scale_log2, -m)); };

    // Of a SIMD's waves the one between the exponentials goes first: it is the way to the next barrier, and the matrix pipe has
    // work queued by the other (not / so, us: 2048 tokens behind 30K 1034 / 998, 4096 from nothing 158 / 149, 2048 of width 64 348 / 326; not for a
    // prefix, whose workgroups run beside streaming ones: 4 tokens each of 64 sequences behind 32K 155 / 158, 256 behind 16K 181 / 180).
    constexpr bool PRIO = !PREFIX;
    el8 kpre[PD];
    int t1, t2, t3;                                      // pages of tiles j + 1, j + 2, j + 3
    // Stage j on the slots of its parity: cur -> P, next <- scores of tile j + 1, if there is one.
    auto stage = [&](auto parity, auto last, Scores &cur, Scores &next, int j) {
        constexpr uint32_t S0 = decltype(parity)::value * SLOT, S1 = SLOT - S0;      // slots of tile j and j + 1
        constexpr bool LAST = decltype(last)::value;
        el8 pr[4];
        float ex[32], sum[2] = {0.f, 0.f};
        auto round_and_sum = [&](auto slot) {            // those of the slot before: nothing waits for a transcendental just issued
            static_range<decltype(slot)::value * EPM, (decltype(slot)::value + 1) * EPM>([&](auto t) {
                pr[t >> 3][t & 7] = (el)ex[t];
                sum[t & 1] += ex[t];
            });
            asm volatile("" : "+v"(sum[0]), "+v"(sum[1]));           // (else the sums are put off, with all they add up kept in registers)
        };
        if constexpr (!LAST) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) next.s[kb][e] = 0.f;
        }
        // (the exponentials stay between these MFMAs: left alone, the compiler moves every other stage's up into the stage
        // before, whose MFMAs have work enough beside them)
        asm volatile("" : "+v"(cur.s[0]), "+v"(cur.s[1]));
        el8 ops[NQK + PD];
#pragma unroll
        for (int n = 0; n < PD; ++n) ops[n] = kpre[n];
        static_for<NQK>([&](auto nc) {
            constexpr int n = decltype(nc)::value;
            if constexpr (!LAST) {
                if constexpr (n + PD < NQK) ops[n + PD] = k_operand(n + PD, S1);
                next.s[n & 1] = mfma16(ops[n], q[n >> 1], next.s[n & 1]);
            }
            static_range<n * EPM, (n + 1) * EPM>([&](auto t) { ex[t] = prob(cur, t); });
            if constexpr (n > 0) round_and_sum(std::integral_constant<int, n - 1>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        round_and_sum(std::integral_constant<int, NQK - 1>{});
        l += sum[0] + sum[1];
        asm volatile("" : "+v"(pr[0]), "+v"(pr[1]), "+v"(pr[2]), "+v"(pr[3]), "+v"(l));
        if constexpr (!LAST) masked(next, j + 1, t1);
        wait_vmcnt<0>();
        wg_barrier();
        if constexpr (PRIO) __builtin_amdgcn_s_setprio(0);
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
            t3 = tile_of(j + 4);
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
        if constexpr (PRIO && !LAST) __builtin_amdgcn_s_setprio(1);
    };

    if (n_tiles > 0) {
        const int t0 = tile_of(0);
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

    if constexpr (PRIO) __builtin_amdgcn_s_setprio(0);

    // ---- results, through the LDS so that rows are written in whole lines ---------------------------------------
    wait_vmcnt<0>();                                     // (the copies of tiles of nothing write their zeros, too)
    wg_barrier();
    l += __shfl_xor(l, 32);
    Args &z = arguments();
    const int end_rows = PREFIX ? z.prefix_rows : z.rows;
    const float f = direct ? normaliser(l) : 1.f;
    constexpr int CH = D / 4;                            // 16-byte chunks of a row of 32-bit results
    float *const ro = reinterpret_cast<float *>(shared.ring) + wave * 32 * D;
#pragma unroll
    for (int y = 0; y < DB; ++y)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int d = D == 128 ? 16 * y + 64 * (c >> 1) + 8 * (c & 1) + 4 * hh : 32 * y + 8 * c + 4 * hh;
            *reinterpret_cast<f32x4 *>(ro + l32 * D + (((d >> 2) ^ (l32 % CH)) << 2)) =
                f32x4{o[y][4 * c] * f, o[y][4 * c + 1] * f, o[y][4 * c + 2] * f, o[y][4 * c + 3] * f};
        }
    const int at_lane = anew(lane);
    if (at_lane < 32) {
        const int row = row0 + wave * 32 + at_lane;
        const Row y = row_of<PREFIX>(end_rows, z.p.group, z.p.seqlen, row, r.b, hk);
        if (direct) {
            if (z.p.lse && y.stored && y.i < qn) z.p.lse[((int64_t)y.b * z.p.seqlen + y.i) * z.p.hq + y.h] = natural_lse(m, l);
        } else if (y.stored)
            (PREFIX ? z.prefix_ml : z.own_ml)[((int64_t)r.slot * z.p.hkv + hk) * end_rows + row] = make_float2(m, l);
    }
    constexpr int AT_ONCE = 64 / CH;                     // rows
    for (int n = at_lane / CH; n < 32; n += AT_ONCE) {
        const int row = row0 + wave * 32 + n, c = at_lane % CH;
        const Row y = row_of<PREFIX>(end_rows, z.p.group, z.p.seqlen, row, r.b, hk);
        const f32x4 v = *reinterpret_cast<const f32x4 *>(ro + n * D + ((c ^ (n % CH)) << 2));
        if (!y.stored) continue;
        if (direct) {
            if (y.i >= qn) continue;
            typedef el el4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<el4 *>(z.p.out + y.b * z.p.osb + y.i * z.p.osn + y.h * z.p.osh + 4 * c) = el4{(el)v[0], (el)v[1], (el)v[2], (el)v[3]};
        } else {
            float *dst = (PREFIX ? z.prefix_o : z.own_o) + (((int64_t)r.slot * z.p.hkv + hk) * end_rows + row) * D;
            *reinterpret_cast<f32x4 *>(dst + 4 * c) = v;
        }
    }
}

// ---- the kernels ------------------------------------------------------------------------------------------
// One launch for the prefix and few rows of own tokens.  Workgroups of a KV head lie hkv apart, so that with 8 of them
// (or a multiple) all that read one head's keys share an XCD's L2.
struct Work {
    bool prefix;
    int hk, x, rg;
};
__device__ __forceinline__ Work work_of(Args &a)
{
    Work w;
    w.hk = blockIdx.x % a.p.hkv;
    int v = blockIdx.x / a.p.hkv;
    const int n = a.prefix_parts * a.prefix_groups;
    w.prefix = v < n;
    if (!w.prefix) v -= n;
    const int groups = w.prefix ? a.prefix_groups : a.groups;
    w.x = v / groups;
    w.rg = groups - 1 - (v - w.x * groups);              // (later rows see more keys: first)
    return w;
}

template <int D, int NRT, bool F16, bool TILED_PREFIX>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) paged_stream_kernel(const Launch)
{
    __shared__ __attribute__((aligned(1024))) union { StreamLds<D, NRT> stream; TileLds<D> tile; } shared;
    const Work w = work_of(arguments());
    if (w.prefix) {
        Args &a = arguments();
        const Range r = prefix_range(a, w.x);
        if constexpr (TILED_PREFIX) tile_range<D, F16, true>(a, r, w.hk, w.rg, shared.tile);
        else stream_range<D, NRT, F16, true>(a, r, w.hk, w.rg, shared.stream);
    } else {
        own_ranges<true>(w.hk, w.x, w.rg, [&](const Range &r) { stream_range<D, NRT, F16, false>(arguments(), r, w.hk, w.rg, shared.stream); });
    }
}

template <int D, bool F16, bool PREFIX>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) paged_tile_kernel(const Launch)
{
    __shared__ __attribute__((aligned(1024))) TileLds<D> shared;
    Args &a = arguments();
    const int hk = blockIdx.x % a.p.hkv, v = blockIdx.x / a.p.hkv, groups = PREFIX ? a.prefix_groups : a.groups;
    const int x = v / groups, rg = groups - 1 - (v - x * groups);          // (later rows see more keys: first)
    if constexpr (PREFIX) tile_range<D, F16, true>(a, prefix_range(a, x), hk, rg, shared);
    else own_ranges<false>(hk, x, rg, [&](const Range &r) { tile_range<D, F16, false>(arguments(), r, hk, rg, shared); });
}

// Ranges joined.  A group of D / 4 lanes (one 16-byte load a lane) takes the ranges of a row of one query head in turn; GPR
// groups share a row: one where there are many rows, all of the workgroup where there are few, and many ranges.
template <int D> constexpr int join_groups() { return 256 / (D / 4); }
template <int D, bool F16, int GPR>
__global__ void __launch_bounds__(256) paged_join_kernel(const Launch)
{
    Args &a = arguments();
    typedef typename Elem<F16>::T el;
    typedef el el4 __attribute__((ext_vector_type(4)));
    constexpr int LANES = D / 4, GROUPS = join_groups<D>();
    __shared__ f32x4 red_o[GPR > 1 ? GROUPS : 1][LANES];
    __shared__ float2 red_ml[GROUPS];
    Params &p = a.p;
    const int group = threadIdx.x / LANES, at_lane = threadIdx.x % LANES;
    const int id = GPR > 1 ? blockIdx.x : blockIdx.x * GROUPS + group, sub = GPR > 1 ? group : 0;
    if (id >= p.batch * p.seqlen * p.hq) return;
    const int t = id / p.hq, h = id - t * p.hq, b = t / p.seqlen, i = t - b * p.seqlen;
    const int2 mine = a.shares ? a.own_ranges[b] : make_int2(b, 1);      // the sequence's ranges
    const int own = mine.y;
    if (i >= queries_of(p, b) || (a.direct && own == 1)) return;         // (written already)
    const int hk = h / p.group, g = h - hk * p.group;
    const int64_t own_at = ((int64_t)mine.x * p.hkv + hk) * a.rows + i * p.group + g;
    const int64_t prefix_at = (int64_t)hk * a.prefix_rows + ((int64_t)b * p.seqlen + i) * p.group + g;
    const int64_t own_step = (int64_t)p.hkv * a.rows, prefix_step = (int64_t)p.hkv * a.prefix_rows;
    const int n = a.prefix_parts + own;
    float m = kNone, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    // (ranges of a group that are requested together; groups that share a row mostly have one or two, and a repeated last range is
    // read again: 1 / 2 / 4 / 8 us, a thousand tokens 9.0 / 8.9 / 9.2 / 9.7, 24 sequences of 300 to 1500 20.9 / 21.1 / 21.4 / 22.4)
    constexpr int AT_ONCE = GPR > 1 ? 2 : 4;
    for (int y0 = sub; y0 < n; y0 += AT_ONCE * GPR) {
        float2 ml[AT_ONCE];
        f32x4 v[AT_ONCE];
#pragma unroll
        for (int c = 0; c < AT_ONCE; ++c) {
            const int y = min(y0 + c * GPR, n - 1);
            const bool pre = y < a.prefix_parts;
            const int64_t at = pre ? prefix_at + y * prefix_step : own_at + (y - a.prefix_parts) * own_step;
            ml[c] = (pre ? a.prefix_ml : a.own_ml)[at];
            if (y0 + c * GPR >= n) ml[c] = make_float2(kNone, 0.f);      // (a repeated last range counts for nothing)
            v[c] = *reinterpret_cast<const f32x4 *>((pre ? a.prefix_o : a.own_o) + at * D + at_lane * 4);
        }
        float mm = m;
#pragma unroll
        for (int c = 0; c < AT_ONCE; ++c) mm = fmaxf(mm, ml[c].x);
        const float f = __builtin_amdgcn_exp2f(m - mm);
        l *= f;
        o *= f;
#pragma unroll
        for (int c = 0; c < AT_ONCE; ++c) {
            const float w = y0 + c * GPR < n ? __builtin_amdgcn_exp2f(ml[c].x - mm) : 0.f;
            l = fmaf(ml[c].y, w, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(v[c][e], w, o[e]);
        }
        m = mm;
    }
    if constexpr (GPR > 1) {
        red_o[group][at_lane] = o;
        if (at_lane == 0) red_ml[group] = make_float2(m, l);
        __syncthreads();
        if (group != 0) return;
#pragma unroll
        for (int y = 0; y < GROUPS; ++y) m = fmaxf(m, red_ml[y].x);
        l = 0.f;
        o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < GROUPS; ++y) {
            const float w = __builtin_amdgcn_exp2f(red_ml[y].x - m);
            l = fmaf(red_ml[y].y, w, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(red_o[y][at_lane][e], w, o[e]);
        }
    }
    const float f = normaliser(l);
    *reinterpret_cast<el4 *>(p.out + b * p.osb + i * p.osn + h * p.osh + at_lane * 4) = el4{(el)(o[0] * f), (el)(o[1] * f), (el)(o[2] * f), (el)(o[3] * f)};
    if (p.lse && at_lane == 0) p.lse[((int64_t)b * p.seqlen + i) * p.hq + h] = natural_lse(m, l);
}

// ---- launch -----------------------------------------------------------------------------------------------
constexpr int kCus = 256;
// Up to that many rows of a unit, one or two 16-row sets of accumulators, are streamed (streamed / with the kernel of many rows, us, 32
// rows: 8 sequences of 2K to 8K tokens 37 / 42, two of 32K 51 / 54, 24 of 700 to 6000 of width 64 25.5 / 32.4, but 64 of 100 to 500 30 / 25;
// 16 rows: 16 of 1K to 4K 31 / 39).  Three sets, and four at width 64, would fit the registers of two waves to a SIMD (212 and 162 of
// 256), four at width 128 would not (48 bytes spilled); 33 rows and more have not been measured in this kernel.
constexpr int kFewRows = 32;
static int64_t up256(int64_t x) { return (x + 255) & ~(int64_t)255; }
static int row_groups(int rows) { return rows <= kFewRows ? 1 : (rows + kTileRows - 1) / kTileRows; }

// How the work is cut up; returns the bytes of workspace.
static int64_t plan(Launch &a, int head_dim)
{
    const PagedParams &p = a.p;
    a.rows = p.seqlen * p.group;
    a.groups = row_groups(a.rows);
    a.direct = p.prefix == 0;
    const int64_t side = (int64_t)p.hkv * a.groups, items = p.batch * side;
    const bool few = a.rows <= kFewRows;
    // Dealt evenly, one workgroup of the streaming kernel to a CU, two of the other; one workgroup to a sequence where sequences
    // fill the chip four times over (twice) anyway, whose results need no joining (dealt / not, us: 64 sequences of 1K to 8K tokens, 512
    // places, 162 / 183, of 2K each 98 / 95; 96 of 300 to 6000, 768, 140 / 155; 128 of 300 to 1500, 1024, 82 / 79; two workgroups of the
    // streaming kernel to a CU: 64 of 1K to 8K 166, two of 128K 188 instead of 185).
    // The least a workgroup gets: a tile to a wave (4 / 8 sub-blocks, us: 16 sequences of 20 to 300 tokens 9.8 / 12.4), six tiles of the kernel of
    // many rows (16 / 24 / 32, us: 64 new tokens of 12 sequences of 134 to 300 23.3 / 17.4 / 17.5, up to 165 of 5 of 250 to 1800 28.0 / 23.9 / 26.4,
    // 32 of 4 of 500 to 2000 30.0 / 28.0 / 29.5, a prompt of 1000 23.4 / 24.4 / 25.2).
    a.min_share = few ? 4 : 24;
    a.near = 8;
    a.shares = p.max_len > 256 && items < (few ? 4 : 2) * kCus ? (int)std::max<int64_t>(1, (few ? 1 : 2) * kCus / side) : 0;
    // A sequence counts as two sub-blocks more than it has, which is what a range's beginning and end take (not / so, us: 16 sequences of
    // 20 to 300 tokens 12.0 / 9.8, 13 of 40 to 350 and two KV heads 10.8 / 9.0, 8 short ones behind 2000 tokens 14.7 / 12.4, 44 of 120 to 640, seven
    // new tokens, 20.1 / 19.0; but 16 of 500, an even number of tiles each, 12.5 / 12.9); few long ones are dealt as they are (two of 32K, 8 new
    // tokens, 50 / 53).
    a.range_cost = 4 * p.batch >= a.shares || p.batch * (int64_t)p.max_len <= (int64_t)a.shares * 16 * kSub ? 2 : 0;
    a.own_slots = a.shares + p.batch;
    if (p.prefix) {
        a.prefix_rows = p.batch * a.rows;
        a.prefix_groups = row_groups(a.prefix_rows);
        const int64_t units = (int64_t)p.hkv * a.prefix_groups;
        // One workgroup of the prefix to a CU leaves the other place to the own tokens, which then arrive while the prefix is
        // multiplied; two multiply faster, which counts where that takes longest (one / two, us: 64 sequences behind 32K 64 / 75,
        // 256 behind 16K 99 / 113; 4 tokens each of 64 behind 32K 165 / 144, two of 256 behind 16K 180 / 173).  The line goes by the products alone:
        // 128 sequences behind 32K have as many as 256 behind 16K and get one workgroup, too, though two would be faster (93 / 90).
        const bool long_products = units * p.prefix > (int64_t)96 * kTileKeys * kCus;
        const int64_t want = std::max<int64_t>(1, (long_products ? 2 : 1) * kCus / units);
        // (at least 64 / 128 / 192 / 256 tokens, us: 62 sequences of 2 tokens behind 1000 22.2 / 22.0 / 19.6 / 21.2, 27 behind 1900 21.3 / 19.5 / 18.5 / 18.7,
        // 98 of width 64 behind 1000 21.8 / 21.6 / 19.9 / 20.4, 2 behind 700 8.1 / 7.9 / 8.4 / 8.9)
        a.prefix_chunk = std::max(192, (int)((p.prefix + want - 1) / want + 63) / 64 * 64);
        a.prefix_parts = (p.prefix + a.prefix_chunk - 1) / a.prefix_chunk;
    }
    const bool joined = a.shares || p.prefix;
    const int64_t own = joined ? (int64_t)a.own_slots * p.hkv * a.rows : 0, prefix = (int64_t)a.prefix_parts * p.hkv * a.prefix_rows;
    unsigned char *at = p.workspace;
    a.own_o = reinterpret_cast<float *>(at);
    a.own_ml = reinterpret_cast<float2 *>(at += up256(own * head_dim * 4));
    a.prefix_o = reinterpret_cast<float *>(at += up256(own * 8));
    a.prefix_ml = reinterpret_cast<float2 *>(at += up256(prefix * head_dim * 4));
    a.own_ranges = reinterpret_cast<int2 *>(at += up256(prefix * 8));
    return at + (a.shares ? up256((int64_t)p.batch * 8) : 0) - p.workspace;
}

size_t paged_workspace_bytes(const PagedParams &p, int head_dim)
{
    Launch a = {};
    a.p = p;
    return (size_t)plan(a, head_dim);
}

template <int D, bool F16> static hipError_t launch(const PagedParams &p, hipStream_t stream)
{
    Launch a = {};
    a.p = p;
    const bool joined = plan(a, D) > 0;
    const unsigned own = (unsigned)((int64_t)(a.shares ? a.shares : p.batch) * a.groups * p.hkv);
    const unsigned prefix = (unsigned)((int64_t)a.prefix_parts * a.prefix_groups * p.hkv);
    const bool tiled_prefix = a.prefix_rows > kFewRows;
    if (a.rows > kFewRows) {
        if (prefix) paged_tile_kernel<D, F16, true><<<prefix, 256, 0, stream>>>(a);
        paged_tile_kernel<D, F16, false><<<own, 256, 0, stream>>>(a);
    } else if (tiled_prefix) {
        if (a.rows <= 16) paged_stream_kernel<D, 1, F16, true><<<prefix + own, 256, 0, stream>>>(a);
        else paged_stream_kernel<D, 2, F16, true><<<prefix + own, 256, 0, stream>>>(a);
    } else {
        if (std::max(a.rows, a.prefix_rows) <= 16) paged_stream_kernel<D, 1, F16, false><<<prefix + own, 256, 0, stream>>>(a);
        else paged_stream_kernel<D, 2, F16, false><<<prefix + own, 256, 0, stream>>>(a);
    }
    if (joined) {
        const int64_t out = (int64_t)p.batch * p.seqlen * p.hq;
        constexpr int GROUPS = join_groups<D>();
        if (out <= 2048) paged_join_kernel<D, F16, GROUPS><<<(unsigned)out, 256, 0, stream>>>(a);
        else paged_join_kernel<D, F16, 1><<<(unsigned)((out + GROUPS - 1) / GROUPS), 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_paged(const PagedParams &p, int head_dim, bool f16, hipStream_t stream)
{
    if (head_dim == 128) return f16 ? launch<128, true>(p, stream) : launch<128, false>(p, stream);
    if (head_dim == 64) return f16 ? launch<64, true>(p, stream) : launch<64, false>(p, stream);
    return hipErrorInvalidValue;
}

}  // namespace bsfa
