// Decode attention over a paged cache, bf16 or 4 bits: one new query per head, a table of pages and a length per sequence.
//
//   out = softmax(scale q K^T) V      S^T = K q^T and O^T = V^T P^T on mma.sync m16n8k16, 16 keys (16 elements of d) as its rows and the up
//                                     to eight queries of a K/V head as its columns
//
// HBM-bound: 4 d (bf16) or 1.125 d (4 bits) bytes per key and K/V head.  Keys as the rows of the tile: a group of up to eight queries costs
// one product per 256 elements of the cache, half of what the queries as 16 rows would (groups of 9 to 16: two).  What bounds the 4-bit form beside the
// bytes is its instructions: an SM has about 400 issue slots in the time HBM takes for 16 keys of a head at d = 128 (2304 bytes).  So
//   * codes become bf16 by one mask (see `nibbles`).  K: the 8 too many are taken off in the products' starting value, -8 sum(q) of the
//     group; V: by one packed subtraction, exact;
//   * K's scale multiplies the products of a group of 32, in fp32; V's is multiplied into the weights, and the product rounded to bf16: the one rounding
//     of a weight (it goes there in two pieces; rounded before, too, the results are off by 0.0029 in place of 0.0023, and
//     the largest case takes 233 us in place of 241);
//   * the page's layout (cache_layout.cuh) is the one in which a lane's codes and scales are 16-byte words: no exchange of any kind.
// Loads.  4 bits: a fifth warp asks for the blocks of a unit by bulk copies, a lane for each of its eight blocks, with the table entries of the next four
// units in its lanes and those behind them on their way; a ring of three units.  bf16: a warp streams its 16 keys at a time through a
// ring of its own (cp.async with the swizzle that ldmatrix wants; no barrier among warps), the entries of its next 32 steps in its lanes.
//
// Work split: a unit is 64 (bf16) or 128 keys of a K/V head, a step of each warp of a CTA.  All units of all sequences, in the order sequence, head, key, are cut into
// equal shares, one per resident team, on the device (the host does not know the lengths): every CTA adds up the lengths and finds its
// teams' shares.  A head that lies in one share is written at once; the teams of the others leave partial results (at most two each), and the last of
// them to come joins them, told by a counter that a one-block kernel in front has cleared; the streaming starts without waiting for that.
// Where there are few heads, one or more clusters take each and join their teams through distributed shared memory (several: the last of them to come
// joins what the others left).  Which of the two: by the estimate in `launch`.
#include "cache_layout.cuh"
#include "ptx.cuh"
#include <algorithm>
#include <cmath>

namespace moa {
namespace {

using namespace ptx;

constexpr int kWarps = 4;            // that compute
enum : uint32_t { PERR_EMPTY = 0x331, PERR_FULL = 0x332 };
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRescale = 8.f;      // weights may exceed 1 by this power of two before the sums are scaled again

struct PagedArgs {
    const __nv_bfloat16 *q;
    const uint8_t *pool;
    const int *table, *lens;
    __nv_bfloat16 *out;
    float *lse, *part_o, *part_ml;
    unsigned int *counters;     // of a share: how many of those that hold the head that begins in it and goes on have left their part
    RopeStride sq;
    long long table_stride, page_stride;
    int B, Hkv, G, pages, page, cap;      // cap: keys that a row of the table has room for
    FastDiv by_page;
    int cl, nc;                 // CTAs of a cluster, clusters of a head; 0: no clusters
    float scale_log2;           // > 0; the sign (or 0) is q's factor, a pair of bf16
    uint32_t sign2;
    unsigned int *status;
};

template <int D, bool kInt4, int NQ>
struct Cfg {
    static constexpr int kTeams = kInt4 ? (NQ == 2 ? 2 : 3) : 1;                       // of kWarps warps, with a share of the work each
    static constexpr int kThreads = 128 * (kTeams + (kInt4 ? 1 : 0));
    static constexpr int kSub = kInt4 ? 2 : 1;                                         // blocks of 16 keys that a warp takes in a step
    static constexpr int kBlocks = kSub * kWarps, kUnitKeys = 16 * kBlocks;
    static constexpr int kBlock = kInt4 ? Block4<D>::kBytes : 16 * D * 4;
    static constexpr int kCtas = kInt4 ? 1 : NQ == 2 || D == 128 ? 2 : 3;              // resident per SM
    static constexpr int kShares = kCtas * kTeams;                                     // per SM
    static constexpr int kStages = kInt4 ? (D == 64 ? 6 : NQ == 2 ? 4 : 3) : D == 128 ? 3 : 4;
    static constexpr int kLd = D + 4;                                                  // floats of a row of the merge
    // shared memory of a team
    static constexpr int offMerge = kStages * kBlocks * kBlock;
    static constexpr int offMl = offMerge + kWarps * 8 * kLd * 4;                      // [warps][8] (maximum, sum)
    static constexpr int offBar = offMl + kWarps * 8 * 8;                              // full, empty [stages], then [stages] words: blocks that hold keys
    static constexpr int offFlag = offBar + kStages * 20 + 4;
    static constexpr int kTeam = (offFlag + 4 + 127) / 128 * 128;
    static constexpr int offScan = kTeams * kTeam;                                     // of the CTA: 16 words of sums, two for each team
    static constexpr int kTotal = offScan + 128;
    static_assert(kCtas * (kTotal + 1024) <= 228 * 1024, "an SM holds kCtas of them, with 1 KB of the system's each (bf16, d = 128: to the byte; one CTA 165 us, two 160)");
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// mma16816 from a starting value of its own: rows g and g + 8 begin at (c0, c1)
__device__ __forceinline__ void mma16816_from(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %10, %11};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}
// Codes as numbers where they lie: a nibble at bits 0..3 or 4..7 of a bf16 whose other bits are zero is c * 2^-133 or c * 2^-129 (the format is
// linear from 0 to twice its least normal number), so one mask makes a pair of them.  What they meet is larger by 2^64: sums of values are 2^-69 or 2^-65 of
// what they stand for and reach into fp32's subnormal numbers, which this file keeps (it is built without flushing them; the same time, and without
// it half of the results below 2^-57 were 0).
constexpr int kCodeExp0 = -133, kCodeExp1 = -129, kLift = 64;
__device__ __forceinline__ uint32_t nibbles(uint32_t w, int i) { return w & (i & 1 ? 0x00f000f0u : 0x000f000fu); }      // w: shifted by 8 for i = 2, 3
__host__ __device__ constexpr float exp2i(int e) { return e < 0 ? 0.5f * exp2i(e + 1) : e > 0 ? 2.f * exp2i(e - 1) : 1.f; }
__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ uint32_t upper(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632); }      // their upper halves
__device__ __forceinline__ float rest(float a) { return a - __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
// The largest bf16 below a > 0 (0 for 0): what it leaves of a is not 0 either, so that both products with an infinite value are infinite
__device__ __forceinline__ float below(float a) { return __uint_as_float((max(__float_as_uint(a), 1u) - 1u) & 0xffff0000u); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

template <int kUnitKeys> __device__ __forceinline__ int units_of(int len) { return len > 0 ? (len + kUnitKeys - 1) / kUnitKeys : 1; }
__device__ __forceinline__ int first_unit(int units, int c, int shares) { return (int)((long long)units * c / shares); }

// Shares, one for each team of the grid: share c is units [first_unit(c), first_unit(c + 1)) of `units`.  Team k of CTA b has share k * gridDim + b, so that
// the first teams of all CTAs come first.
struct Share {
    int units, shares, c, u0, u1, b, before;      // b: the sequence that holds u0; before: units in front of it
};
template <class C> __device__ __forceinline__ Share find_share(const PagedArgs &a, const int *lens, int *scan, int team)
{
    constexpr int kThreads = C::kThreads, kAll = kThreads / 32;
    static_assert(kAll <= 16, "a warp's sum each");
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    Share s;
    int sum = 0, first = 0;
    for (int b = tid; b < a.B; b += kThreads) {
        const int n = units_of<C::kUnitKeys>(min(lens[b], a.cap));
        if (b == tid) first = n;
        sum += n;
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) scan[warp] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kAll; ++w) sum += scan[w];
    s.units = sum * a.Hkv;
    s.shares = min((int)gridDim.x * C::kTeams, s.units);
    auto begin_of = [&](int c) { return c < s.shares ? first_unit(s.units, c, s.shares) : s.units; };
    int row[C::kTeams], carry = 0;      // where each team's share begins, in units of one head (all heads have the same)
#pragma unroll
    for (int k = 0; k < C::kTeams; ++k) row[k] = begin_of(k * (int)gridDim.x + (int)blockIdx.x) / a.Hkv;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid, n = b0 == 0 ? first : b < a.B ? units_of<C::kUnitKeys>(min(lens[b], a.cap)) : 0;
        int incl = n;
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        __syncthreads();
        if (lane == 31) scan[warp] = incl;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < kAll; ++w) {
            if (w < warp) incl += scan[w];
            all += scan[w];
        }
        incl += carry;
#pragma unroll
        for (int k = 0; k < C::kTeams; ++k)
            if (incl - n <= row[k] && row[k] < incl) { scan[16 + 2 * k] = b; scan[17 + 2 * k] = incl - n; }
        carry += all;
        if (carry > row[C::kTeams - 1]) break;      // (the same in every thread; the last team's is the last)
    }
    __syncthreads();
    s.c = team * (int)gridDim.x + (int)blockIdx.x;
    s.u0 = begin_of(s.c);
    s.u1 = begin_of(s.c + 1);
    s.b = s.u0 < s.u1 ? scan[16 + 2 * team] : 0;
    s.before = s.u0 < s.u1 ? scan[17 + 2 * team] * a.Hkv : 0;
    return s;
}

// With clusters: CTA rank r of a head's j-th cluster, team k: part (j * cl + r) * kTeams + k of the head's units
template <class C> __device__ __forceinline__ Share cluster_share(const PagedArgs &a, const int *lens, int team)
{
    Share s;
    const int cluster = (int)blockIdx.x / a.cl, head = cluster / a.nc, parts = a.nc * a.cl * C::kTeams;
    const int part = ((cluster - head * a.nc) * a.cl + (int)cluster_ctarank()) * C::kTeams + team;
    s.b = head / a.Hkv;
    const int n = units_of<C::kUnitKeys>(min(lens[s.b], a.cap));
    s.units = n * a.Hkv;
    s.shares = parts;
    s.c = part;
    s.before = 0;
    s.u0 = (head - s.b * a.Hkv) * n + first_unit(n, part, parts);
    s.u1 = (head - s.b * a.Hkv) * n + first_unit(n, part + 1, parts);
    return s;
}

// A place in a share: unit t of head h of sequence b, whose length is len
template <class C> struct Place {
    int b, h, t, len, end;      // end: units of a head of the sequence
    __device__ __forceinline__ void set(int seq, int head, int unit, int n)
    {
        b = seq; h = head; t = unit; len = n; end = units_of<C::kUnitKeys>(n);
    }
};
__device__ __forceinline__ int length_of(const PagedArgs &a, const int *lens, int b) { return b < a.B ? max(0, min(lens[b], a.cap)) : 0; }
// Where block `block` of unit t begins (4 bits: the block, bf16: the row of K), as an offset from the pool; -1: the table has no such page
template <int D, bool kInt4, class C>
__device__ __forceinline__ long long block_offset(const PagedArgs &a, const int *table, int b, int h, int t, int block)
{
    const int key = t * C::kUnitKeys + 16 * block;
    if (key >= a.cap || b >= a.B) return -1;
    const int at = (int)a.by_page.div((uint32_t)key), in = key - at * a.page, pg = table[b * a.table_stride + at];
    if ((unsigned)pg >= (unsigned)a.pages) return -1;
    return pg * a.page_stride + (kInt4 ? block4<D>(a.page, h, in / kBlockKeys) : row16(a.page, D, h, 0, in));
}

// What a warp knows of a head: its queries as B operands (times the scale's sign), and, over the keys it has seen, O^T and the weights' sum.
// Weights are 2^(scale * product - ref); a product above `top` moves ref (top = -inf: nothing seen yet).  4 bits: products of scores come out
// lowered, the weights and their sum are raised by 2^kUp.
template <int D, bool kInt4, int NQ>
struct HeadState {
    static constexpr int kG = D / 32, kNO = D / 16, kSub = Cfg<D, kInt4, NQ>::kSub;
    static constexpr float kUp = kInt4 ? (float)kLift : 0.f;
    // A weight as a bf16 and what that leaves, another.  4 bits: its product with V's scale is rounded once.  bf16: a product each, nothing is rounded
    // to bf16 but the result (error against 64 bits 0.0023 -> 0.0017; B8 H32/8 n32768 160.3 -> 161.1 us, H32/4 87.4 -> 89.1).  With groups of 9 to 16, which
    // compute for longer, that would be 8 to 13 % (B8 H32/2 n32768 53.2 -> 60.3 us): they round a weight, as 4 bits do its product (both
    // pieces of that one: n131072 250 -> 283 us).
    static constexpr bool kPieces = kInt4 || NQ == 1;
    uint32_t qf[NQ][kInt4 ? 4 * kG : D / 8];
    float bias[NQ][kInt4 ? kG : 1][2];      // 4 bits: the products' starting values
    float o[NQ][kNO][4], ref[NQ][2], top[NQ][2], l[NQ][2];

    __device__ __forceinline__ void begin(const PagedArgs &a, const __nv_bfloat16 *q, int b, int h, int lane)
    {
        const int g = lane / 4, t4 = lane % 4;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int row = 8 * n + g;
            const __nv_bfloat16 *src = q + a.sq.at(b, h * a.G + row);
            if constexpr (kInt4) {
#pragma unroll
                for (int y = 0; y < kG; ++y) {
                    uint4 v = row < a.G ? *reinterpret_cast<const uint4 *>(src + 32 * y + 8 * t4) : make_uint4(0u, 0u, 0u, 0u);
                    v.x = mul2(v.x, a.sign2); v.y = mul2(v.y, a.sign2); v.z = mul2(v.z, a.sign2); v.w = mul2(v.w, a.sign2);
                    float s = ((low_bf16(v.x) + high_bf16(v.x)) + (low_bf16(v.y) + high_bf16(v.y))) + ((low_bf16(v.z) + high_bf16(v.z)) + (low_bf16(v.w) + high_bf16(v.w)));
                    // (even words meet nibbles 0 and 2, odd ones nibbles 1 and 3, which weigh 16 times as much)
                    const uint32_t up0 = 0x5f805f80u + (4u << 7) * 0x10001u, up1 = 0x5f805f80u;      // 2^68, 2^64
                    qf[n][4 * y] = mul2(v.x, up0); qf[n][4 * y + 1] = mul2(v.y, up1); qf[n][4 * y + 2] = mul2(v.z, up0); qf[n][4 * y + 3] = mul2(v.w, up1);
                    s += __shfl_xor_sync(0xffffffffu, s, 1);
                    s += __shfl_xor_sync(0xffffffffu, s, 2);
                    s *= -8.f * exp2i(kCodeExp1 + kLift);
                    bias[n][y][0] = __shfl_sync(0xffffffffu, s, 8 * t4);
                    bias[n][y][1] = __shfl_sync(0xffffffffu, s, 8 * t4 + 4);
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 8; ++i) qf[n][i] = mul2(row < a.G ? *reinterpret_cast<const uint32_t *>(src + 8 * i + 2 * t4) : 0u, a.sign2);
            }
            ref[n][0] = ref[n][1] = -kUp;
            top[n][0] = top[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.f;
#pragma unroll
            for (int i = 0; i < kNO; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
        }
    }

    // scores of a block of 16 keys: rows g and g + 8 of the tile are keys, columns 2 t4 and 2 t4 + 1 queries
    __device__ __forceinline__ void scores(float (&sc)[NQ][4], uint32_t blk, int lane) const
    {
        const int g = lane / 4, t4 = lane % 4;
        if constexpr (kInt4) {
            uint32_t k0[kG], k1[kG], ks[kG];      // a lane's words are eight elements of each group
            if constexpr (D == 128) {
                const uint4 x = lds128(blk + g * 64 + t4 * 16), y = lds128(blk + (g + 8) * 64 + t4 * 16), z = lds128(blk + Block4<D>::offKS + g * 16);
                k0[0] = x.x; k0[1] = x.y; k0[2] = x.z; k0[3] = x.w;
                k1[0] = y.x; k1[1] = y.y; k1[2] = y.z; k1[3] = y.w;
                ks[0] = z.x; ks[1] = z.y; ks[2] = z.z; ks[3] = z.w;
            } else {
                const uint2 x = lds64(blk + g * 32 + t4 * 8), y = lds64(blk + (g + 8) * 32 + t4 * 8), z = lds64(blk + Block4<D>::offKS + g * 8);
                k0[0] = x.x; k0[1] = x.y;
                k1[0] = y.x; k1[1] = y.y;
                ks[0] = z.x; ks[1] = z.y;
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
            for (int y = 0; y < kG; ++y) {
                const uint32_t h0 = k0[y] >> 8, h1 = k1[y] >> 8;
                const uint32_t lo[4] = {nibbles(k0[y], 0), nibbles(k1[y], 0), nibbles(k0[y], 1), nibbles(k1[y], 1)};
                const uint32_t hi[4] = {nibbles(h0, 2), nibbles(h1, 2), nibbles(h0, 3), nibbles(h1, 3)};
                // scales: words [row g: groups 0 1, 2 3][row g + 8: 0 1, 2 3]
                const uint32_t w0 = ks[y / 2], w1 = ks[kG / 2 + y / 2];
                const float s0 = y % 2 ? high_bf16(w0) : low_bf16(w0), s1 = y % 2 ? high_bf16(w1) : low_bf16(w1);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    float c[4];
                    mma16816_from(c, lo, qf[n][4 * y], qf[n][4 * y + 1], bias[n][y][0], bias[n][y][1]);
                    mma16816(c, hi, qf[n][4 * y + 2], qf[n][4 * y + 3]);
                    sc[n][0] = fmaf(s0, c[0], sc[n][0]);
                    sc[n][1] = fmaf(s0, c[1], sc[n][1]);
                    sc[n][2] = fmaf(s1, c[2], sc[n][2]);
                    sc[n][3] = fmaf(s1, c[3], sc[n][3]);
                }
            }
        } else {
            float odd[NQ][4];
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[n][e] = odd[n][e] = 0.f;
            const int r = (lane / 8 & 1) * 8 + lane % 8;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int c = 2 * i + lane / 16;
                uint32_t ka[4];
                ldmatrix4(ka, blk + r * (2 * D) + ((c & ~7) | ((c ^ r) & 7)) * 16);
#pragma unroll
                for (int n = 0; n < NQ; ++n) mma16816(i % 2 ? odd[n] : sc[n], ka, qf[n][2 * i], qf[n][2 * i + 1]);
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[n][e] += odd[n][e];
        }
    }

    // O^T += V^T P^T of a block; keys of it from `in` on do not count (their weights are 0; their scales may not be numbers)
    __device__ __forceinline__ void values(const uint32_t (&pb)[NQ][2], const uint32_t (&pr)[NQ][2], uint32_t blk, int lane, bool ragged, int in)
    {
        const int t4 = lane % 4;
        if constexpr (kInt4) {
            uint32_t va[D / 64][4], vs[kG][2];      // [h][key 2 t, 2 t + 1, 2 t + 8, 2 t + 9]
            const uint32_t vt = blk + Block4<D>::offV, vsc = blk + Block4<D>::offVS;
            if constexpr (D == 128) {
                const uint4 x = lds128(vt + lane * 16), y = lds128(vt + 512 + lane * 16), z = lds128(vsc + t4 * 32), w = lds128(vsc + t4 * 32 + 16);
                va[0][0] = x.x; va[1][0] = x.y; va[0][1] = x.z; va[1][1] = x.w;
                va[0][2] = y.x; va[1][2] = y.y; va[0][3] = y.z; va[1][3] = y.w;
                vs[0][0] = z.x; vs[0][1] = z.y; vs[1][0] = z.z; vs[1][1] = z.w;
                vs[2][0] = w.x; vs[2][1] = w.y; vs[3][0] = w.z; vs[3][1] = w.w;
            } else {
                const uint2 x = lds64(vt + lane * 8), y = lds64(vt + 256 + lane * 8);
                const uint4 z = lds128(vsc + t4 * 16);
                va[0][0] = x.x; va[0][1] = x.y; va[0][2] = y.x; va[0][3] = y.y;
                vs[0][0] = z.x; vs[0][1] = z.y; vs[1][0] = z.z; vs[1][1] = z.w;
            }
            if (ragged) {
                const int k = 2 * t4;
                const uint32_t m0 = (k < in ? 0xffffu : 0u) | (k + 1 < in ? 0xffff0000u : 0u), m1 = (k + 8 < in ? 0xffffu : 0u) | (k + 9 < in ? 0xffff0000u : 0u);
#pragma unroll
                for (int y = 0; y < kG; ++y) { vs[y][0] &= m0; vs[y][1] &= m1; }
            }
#pragma unroll
            for (int y = 0; y < kG; ++y) {
                const uint32_t sel = y % 2 ? 0x7632u : 0x5410u;
                const uint32_t w01 = __byte_perm(va[y / 2][0], va[y / 2][1], sel), w23 = __byte_perm(va[y / 2][2], va[y / 2][3], sel);
                uint32_t b0[NQ], b1[NQ];
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    b0[n] = fma2(pb[n][0], vs[y][0], mul2(pr[n][0], vs[y][0]));
                    b1[n] = fma2(pb[n][1], vs[y][1], mul2(pr[n][1], vs[y][1]));
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t x01 = u ? w01 >> 8 : w01, x23 = u ? w23 >> 8 : w23;
                    uint32_t v[4];
                    v[0] = add2(nibbles(x01, 0), 0x80088008u);          // - 8
                    v[1] = add2(nibbles(x01, 1), 0x80808080u);
                    v[2] = add2(nibbles(x23, 0), 0x80088008u);
                    v[3] = add2(nibbles(x23, 1), 0x80808080u);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) mma16816(o[n][2 * y + u], v, b0[n], b1[n]);
                }
            }
        } else {
            const int r = (lane / 16) * 8 + lane % 8;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int c = 2 * i + (lane / 8 & 1);
                uint32_t v[4];
                ldmatrix4_trans(v, blk + 32 * D + r * (2 * D) + ((c & ~7) | ((c ^ r) & 7)) * 16);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    mma16816(o[n][i], v, pb[n][0], pb[n][1]);
                    if constexpr (kPieces) mma16816(o[n][i], v, pr[n][0], pr[n][1]);
                }
            }
        }
    }

    // A step: kSub blocks at `st`; `here`: which of them hold keys (a bit each), `left`: keys of the sequence from the first of them on
    __device__ __forceinline__ void step(uint32_t st, uint32_t here, int left, float scale, float margin, int lane)
    {
        constexpr int kBlock = Cfg<D, kInt4, NQ>::kBlock;
        constexpr uint32_t kAll = (1u << kSub) - 1;
        const int g = lane / 4;
        float sc[kSub][NQ][4];
#pragma unroll
        for (int s = 0; s < kSub; ++s) scores(sc[s], st + s * kBlock, lane);
        // keys past the end, and blocks that are not there (their stage holds anything)
        const bool ragged = left < 16 * kSub || here != kAll;
        if (ragged) {
#pragma unroll
            for (int s = 0; s < kSub; ++s) {
                const int in = here >> s & 1 ? left - 16 * s : 0;
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (g + 8 * (e / 2) >= in) sc[s][n][e] = -INFINITY;
            }
        }
        bool grow = false;
        float mx[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mx[n][e] = fmaxf(sc[0][n][e], sc[0][n][2 + e]);
#pragma unroll
                for (int s = 1; s < kSub; ++s) mx[n][e] = fmaxf(mx[n][e], fmaxf(sc[s][n][e], sc[s][n][2 + e]));
                grow = grow || mx[n][e] > top[n][e];
            }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float m = mx[n][e];
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                    const float to = fmaf(m, scale, -kUp);
                    if (m > -INFINITY && (top[n][e] == -INFINITY || to > ref[n][e])) {
                        const float f = top[n][e] == -INFINITY ? 1.f : ex2(ref[n][e] - to);      // (nothing seen: the sums are 0)
                        ref[n][e] = to;
                        top[n][e] = m + margin;
                        l[n][e] *= f;
#pragma unroll
                        for (int i = 0; i < kNO; ++i) { o[n][i][e] *= f; o[n][i][2 + e] *= f; }
                    }
                }
        }
        uint32_t pb[kSub][NQ][2], pr[kSub][NQ][2];
#pragma unroll
        for (int s = 0; s < kSub; ++s)
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const float p0 = ex2(fmaf(sc[s][n][0], scale, -ref[n][0])), p1 = ex2(fmaf(sc[s][n][1], scale, -ref[n][1]));
                const float p2 = ex2(fmaf(sc[s][n][2], scale, -ref[n][0])), p3 = ex2(fmaf(sc[s][n][3], scale, -ref[n][1]));
                l[n][0] += p0 + p2;
                l[n][1] += p1 + p3;
                if constexpr (kPieces && !kInt4) {
                    const float h0 = below(p0), h1 = below(p1), h2 = below(p2), h3 = below(p3);
                    pb[s][n][0] = transpose8(upper(h0, h1));
                    pb[s][n][1] = transpose8(upper(h2, h3));
                    pr[s][n][0] = transpose8(pack_bf16(p0 - h0, p1 - h1));
                    pr[s][n][1] = transpose8(pack_bf16(p2 - h2, p3 - h3));
                } else if constexpr (kPieces) {
                    pb[s][n][0] = transpose8(upper(p0, p1));
                    pb[s][n][1] = transpose8(upper(p2, p3));
                    pr[s][n][0] = transpose8(pack_bf16(rest(p0), rest(p1)));
                    pr[s][n][1] = transpose8(pack_bf16(rest(p2), rest(p3)));
                } else {
                    pb[s][n][0] = transpose8(pack_bf16(p0, p1));
                    pb[s][n][1] = transpose8(pack_bf16(p2, p3));
                }
            }
#pragma unroll
        for (int s = 0; s < kSub; ++s) values(pb[s], pr[s], st + s * kBlock, lane, ragged, here >> s & 1 ? left - 16 * s : 0);
    }

    // Eight queries (the n-th eight) of this warp into the merge: rows of kLd floats, and (maximum, sum) of each
    __device__ __forceinline__ void leave(int n, int rows, float *merge, float2 *ml, int warp, int lane) const
    {
        constexpr int kLd = Cfg<D, kInt4, NQ>::kLd;
        const int g = lane / 4, t4 = lane % 4;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float lt = l[n][e];
            lt += __shfl_xor_sync(0xffffffffu, lt, 4);
            lt += __shfl_xor_sync(0xffffffffu, lt, 8);
            lt += __shfl_xor_sync(0xffffffffu, lt, 16);
            const int r = 2 * t4 + e;
            if (r < rows) {
                float *row = merge + (warp * 8 + r) * kLd;
#pragma unroll
                for (int i = 0; i < kNO; ++i) {
                    if constexpr (kInt4) {
                        constexpr float k0 = exp2i(-kCodeExp0 - kLift), k1 = exp2i(-kCodeExp1 - kLift);
                        if (i % 2 == 0)
                            *reinterpret_cast<float4 *>(row + 16 * i + 4 * g) =
                                make_float4(k0 * o[n][i][e], k1 * o[n][i][2 + e], k0 * o[n][i + 1][e], k1 * o[n][i + 1][2 + e]);
                    } else {
                        row[16 * i + g] = o[n][i][e];
                        row[16 * i + 8 + g] = o[n][i][2 + e];
                    }
                }
                if (g == 0) ml[warp * 8 + r] = make_float2(top[n][e] == -INFINITY ? -INFINITY : ref[n][e] + kUp, lt * exp2i(-(int)kUp));
            }
        }
    }
};

// The end of a segment of a head (the warps of a team, all of them): their results joined, eight queries at a time, and written: the head's result
// (whole), or a partial one; with clusters, rows of kLd floats (sums, then maximum and weights' sum) over the team's ring, which is done
template <int D, bool kInt4, int NQ, bool kClusters>
__device__ __forceinline__ void join(const PagedArgs &a, const HeadState<D, kInt4, NQ> &s, uint8_t *smem, int team, int head, bool whole, int slot)
{
    using C = Cfg<D, kInt4, NQ>;
    constexpr int kJoin = 32 * kWarps;
    float *merge = reinterpret_cast<float *>(smem + C::offMerge);
    float2 *ml = reinterpret_cast<float2 *>(smem + C::offMl);
    const int tid = threadIdx.x % kJoin;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int rows = min(8, a.G - 8 * n);
        named_barrier(1 + team, kJoin);                // (the join before has been read)
        s.leave(n, rows, merge, ml, tid / 32, tid % 32);
        named_barrier(1 + team, kJoin);
        for (int idx = tid; idx < rows * (D / 4); idx += kJoin) {
            const int r = idx / (D / 4), c = 4 * (idx % (D / 4));
            float mt = -INFINITY, ls = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) mt = fmaxf(mt, ml[w * 8 + r].x);
            const float ref = mt == -INFINITY ? 0.f : mt;
            float4 ot = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float2 x = ml[w * 8 + r];
                const float f = ex2(x.x - ref);
                const float4 v = *reinterpret_cast<const float4 *>(merge + (w * 8 + r) * C::kLd + c);
                ls = fmaf(x.y, f, ls);
                ot.x = fmaf(v.x, f, ot.x); ot.y = fmaf(v.y, f, ot.y); ot.z = fmaf(v.z, f, ot.z); ot.w = fmaf(v.w, f, ot.w);
            }
            if constexpr (kClusters) {
                float *row = reinterpret_cast<float *>(smem) + (8 * n + r) * C::kLd;
                *reinterpret_cast<float4 *>(row + c) = ot;
                if (c == 0) *reinterpret_cast<float2 *>(row + D) = make_float2(mt, ls);
            } else if (whole) {
                const size_t at = (size_t)head * a.G + 8 * n + r;
                const float inv = ls == 0.f ? 0.f : 1.f / ls;
                *reinterpret_cast<uint2 *>(a.out + at * D + c) = make_uint2(pack_bf16(ot.x * inv, ot.y * inv), pack_bf16(ot.z * inv, ot.w * inv));
                if (a.lse && c == 0) a.lse[at] = ls == 0.f ? -INFINITY : (mt + __log2f(ls)) * kLn2;
            } else {
                const size_t at = (size_t)slot * a.G + 8 * n + r;
                *reinterpret_cast<float4 *>(a.part_o + at * D + c) = ot;
                if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(mt, ls);
            }
        }
    }
}

// The share that holds unit u
__device__ __forceinline__ int share_of(const Share &sh, int u)
{
    int c = (int)((long long)u * sh.shares / sh.units);
    while (first_unit(sh.units, c + 1, sh.shares) <= u) ++c;
    return c;
}

// Four elements of a query, from c on, of `parts` partial results: slot(k) says where part k is; kBatch of them on their way.  Thread `lane` of the kLanes
// (neighbours in a warp) that share them; all of them get the result.
struct Joined {
    float m, l;
    float4 o;
};
template <int D, int kLanes, int kBatch, class Slot>
__device__ __forceinline__ Joined join_parts(const PagedArgs &a, int g, int c, int parts, int lane, Slot slot)
{
    float mt = -INFINITY, ls = 0.f;
    float4 ot = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = lane; k0 < parts; k0 += kLanes * kBatch) {
        float2 ml[kBatch];
        float4 v[kBatch];
        float mn = mt;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const bool there = k0 + u * kLanes < parts;
            const size_t at = (size_t)slot(k0 + u * kLanes) * a.G + g;
            ml[u] = there ? __ldcg(reinterpret_cast<const float2 *>(a.part_ml + at * 2)) : make_float2(-INFINITY, 0.f);
            v[u] = there ? __ldcg(reinterpret_cast<const float4 *>(a.part_o + at * D + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) mn = fmaxf(mn, ml[u].x);
        const float ref = mn == -INFINITY ? 0.f : mn, b = ex2(mt - ref);
        mt = mn;
        ls *= b;
        ot.x *= b; ot.y *= b; ot.z *= b; ot.w *= b;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const float f = ex2(ml[u].x - ref);
            ls = fmaf(ml[u].y, f, ls);
            ot.x = fmaf(v[u].x, f, ot.x); ot.y = fmaf(v[u].y, f, ot.y); ot.z = fmaf(v[u].z, f, ot.z); ot.w = fmaf(v[u].w, f, ot.w);
        }
    }
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) {
        // (both sides on the same reference: their sums add)
        const float mn = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o)), b = ex2(mt - (mn == -INFINITY ? 0.f : mn));
        mt = mn;
        ls *= b;
        ot.x *= b; ot.y *= b; ot.z *= b; ot.w *= b;
        ls += __shfl_xor_sync(0xffffffffu, ls, o);
        ot.x += __shfl_xor_sync(0xffffffffu, ot.x, o); ot.y += __shfl_xor_sync(0xffffffffu, ot.y, o);
        ot.z += __shfl_xor_sync(0xffffffffu, ot.z, o); ot.w += __shfl_xor_sync(0xffffffffu, ot.w, o);
    }
    return Joined{mt, ls, ot};
}
template <int D>
__device__ __forceinline__ void write_result(const PagedArgs &a, int head, int g, int c, const Joined &r)
{
    const size_t at = (size_t)head * a.G + g;
    const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
    *reinterpret_cast<uint2 *>(a.out + at * D + c) = make_uint2(pack_bf16(r.o.x * inv, r.o.y * inv), pack_bf16(r.o.z * inv, r.o.w * inv));
    if (a.lse && c == 0) a.lse[at] = r.l == 0.f ? -INFINITY : (r.m + __log2f(r.l)) * kLn2;
}

// A head that lies in several shares, ca to cb: the team that leaves its part last joins them all (nobody waits for anyone).
template <int D, class C>
__device__ __forceinline__ void last_joins(const PagedArgs &a, int team, int head, int ca, int cb, unsigned int *flag)
{
    constexpr int kJoin = 32 * kWarps;
    const int tid = threadIdx.x % kJoin;
    // the fences of the thread that counts order what the barriers in front of and behind it have gathered: the team's part before the count, the
    // other teams' parts, if it is the last, before the reads
    named_barrier(1 + team, kJoin);
    if (tid == 0) {
        __threadfence();
        *flag = atomicAdd(a.counters + ca, 1u);
        __threadfence();
    }
    named_barrier(1 + team, kJoin);
    if (*flag != (unsigned)(cb - ca)) return;
    for (int idx = tid; idx < a.G * (D / 4); idx += kJoin) {
        const int g = idx / (D / 4), c = 4 * (idx % (D / 4));
        write_result<D>(a, head, g, c, join_parts<D, 1, 4>(a, g, c, cb - ca + 1, 0, [&](int k) { return 2 * (ca + k) + (k == 0 ? 1 : 0); }));
    }
}

// The segments of a share in turn: `next` makes a step of this warp with the head's state
template <int D, bool kInt4, int NQ, bool kClusters, class Next>
__device__ __forceinline__ void walk(const PagedArgs &a, const Share &sh, Place<Cfg<D, kInt4, NQ>> use, const __nv_bfloat16 *q, const int *lens, uint8_t *smem, int team, Next next)
{
    using C = Cfg<D, kInt4, NQ>;
    const int count = sh.u1 - sh.u0, lane = threadIdx.x % 32;
    int done = 0;
    HeadState<D, kInt4, NQ> s;
    if constexpr (kClusters) {
        s.begin(a, q, use.b, use.h, lane);
        for (; done < count; ++done, ++use.t) next(s, use);
        cp_wait<0>();
        join<D, kInt4, NQ, true>(a, s, smem, team, 0, false, 0);
    } else {
        while (done < count) {
            const int first = use.t, steps = min(use.end - use.t, count - done), head = use.b * a.Hkv + use.h;
            s.begin(a, q, use.b, use.h, lane);
            for (int i = 0; i < steps; ++i, ++done, ++use.t) next(s, use);
            const bool whole = first == 0 && use.t == use.end;
            join<D, kInt4, NQ, false>(a, s, smem, team, head, whole, 2 * sh.c + (first == 0 ? 1 : 0));
            if (!whole) {
                // the head's first and last unit, and whose shares those are in
                const int next_unit = sh.u0 + done;
                last_joins<D, C>(a, team, head, first == 0 ? sh.c : share_of(sh, next_unit - use.t),
                                 use.t == use.end ? sh.c : share_of(sh, next_unit - use.t + use.end - 1), reinterpret_cast<unsigned int *>(smem + C::offFlag));
            }
            if (use.t == use.end) {
                int b = use.b, h = use.h + 1;
                if (h == a.Hkv) { h = 0; ++b; }
                use.set(b, h, 0, b == use.b ? use.len : length_of(a, lens, b));
            }
        }
    }
}

// A cluster's teams joined through distributed shared memory.  Each CTA makes a contiguous part of the head's elements, four of them in eight lanes: lane k
// reads the rows of CTA k's teams.  (One CTA that read all of them took 3800 cycles for 24 teams, G = 4.)  `tid` of the `threads` of this CTA that compute.
// Between two barriers of the cluster: every thread of it calls them.
template <int D, bool kInt4, int NQ>
__device__ __forceinline__ void combine(const PagedArgs &a, uint8_t *shared, int tid, int threads)
{
    using C = Cfg<D, kInt4, NQ>;
    const int cluster = (int)blockIdx.x / a.cl, rank = (int)cluster_ctarank(), all = a.G * (D / 4), k = tid % 8;
    const int first = all * rank / a.cl, last = all * (rank + 1) / a.cl;
    const uint32_t base = smem_u32(shared);
    for (int i0 = first; i0 < last; i0 += threads / 8) {       // (whole warps: the exchanges below)
        const int idx = i0 + tid / 8, r = idx / (D / 4), c = 4 * (idx % (D / 4));
        const bool in = idx < last;
        float2 ml[C::kTeams];
        float4 v[C::kTeams];
        float mt = -INFINITY;
#pragma unroll
        for (int j = 0; j < C::kTeams; ++j) {
            ml[j] = make_float2(-INFINITY, 0.f);
            v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (in && k < a.cl) {
                const uint32_t row = mapa_u32(base + j * C::kTeam + r * (4 * C::kLd), (uint32_t)k);
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(ml[j].x), "=f"(ml[j].y) : "r"(row + 4 * D) : "memory");
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[j].x), "=f"(v[j].y), "=f"(v[j].z), "=f"(v[j].w) : "r"(row + 4 * c) : "memory");
            }
        }
#pragma unroll
        for (int j = 0; j < C::kTeams; ++j) mt = fmaxf(mt, ml[j].x);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
        const float ref = mt == -INFINITY ? 0.f : mt;
        float ls = 0.f;
        float4 ot = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < C::kTeams; ++j) {
            const float f = ex2(ml[j].x - ref);
            ls = fmaf(ml[j].y, f, ls);
            ot.x = fmaf(v[j].x, f, ot.x); ot.y = fmaf(v[j].y, f, ot.y); ot.z = fmaf(v[j].z, f, ot.z); ot.w = fmaf(v[j].w, f, ot.w);
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
            ls += __shfl_xor_sync(0xffffffffu, ls, o);
            ot.x += __shfl_xor_sync(0xffffffffu, ot.x, o); ot.y += __shfl_xor_sync(0xffffffffu, ot.y, o);
            ot.z += __shfl_xor_sync(0xffffffffu, ot.z, o); ot.w += __shfl_xor_sync(0xffffffffu, ot.w, o);
        }
        if (in && k == 0) {
            if (a.nc == 1) {
                write_result<D>(a, cluster, r, c, Joined{mt, ls, ot});
            } else {
                const size_t at = (size_t)cluster * a.G + r;
                *reinterpret_cast<float4 *>(a.part_o + at * D + c) = ot;
                if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(mt, ls);
            }
        }
    }
}

// The end of a cluster kernel, for every thread of the cluster: the teams' rows joined, and where a head has several clusters, their partial results by the
// last of them to come, all its CTAs.  `flag` lies behind what combine() reads.  Threads that only load (tid < 0) keep the barriers company.
template <int D, bool kInt4, int NQ>
__device__ __forceinline__ void finish_clusters(const PagedArgs &a, uint8_t *shared, unsigned int *flag, int tid, int threads)
{
    cluster_sync_all();
    if (tid >= 0) combine<D, kInt4, NQ>(a, shared, tid, threads);
    __syncwarp();
    cluster_sync_all();                                        // nobody leaves while another CTA may still read its shared memory
    if (a.nc == 1) return;
    const int head = (int)blockIdx.x / (a.cl * a.nc), rank = (int)cluster_ctarank();
    if (tid == 0 && rank == 0) {                               // (the fences: as in last_joins)
        __threadfence();
        *flag = atomicAdd(a.counters + head, 1u);
        __threadfence();
    }
    __syncwarp();
    cluster_sync_all();
    unsigned int came;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(came) : "r"(mapa_u32(smem_u32(flag), 0u)) : "memory");
    __syncwarp();
    cluster_sync_all();
    if (tid < 0 || came != (unsigned)(a.nc - 1)) return;
    const int all = a.G * (D / 4), first = all * rank / a.cl, last = all * (rank + 1) / a.cl;
    for (int i0 = first; i0 < last; i0 += threads / 4) {       // (whole warps: the exchanges)
        const int idx = i0 + tid / 4, at = min(idx, last - 1), g = at / (D / 4), c = 4 * (at % (D / 4));
        const Joined r = join_parts<D, 4, 4>(a, g, c, a.nc, tid % 4, [&](int k) { return head * a.nc + k; });
        if (idx < last && tid % 4 == 0) write_result<D>(a, head, g, c, r);
    }
}

template <int D, int NQ, bool kClusters>
__global__ void __launch_bounds__((Cfg<D, true, NQ>::kThreads), (Cfg<D, true, NQ>::kCtas)) paged_decode4_kernel(const PagedArgs a)
{
    using C = Cfg<D, true, NQ>;
    constexpr int S = C::kStages, kUnit = C::kBlocks * C::kBlock;
    // registers of a thread that computes and of one that loads: 128 (384 threads: 168) at launch, 3 x 160 + 32 = 4 x 128, 2 x 224 + 56 = 3 x 168
    constexpr int kUseRegs = NQ == 2 ? 224 : 160, kLoadRegs = NQ == 2 ? 56 : 32;
    extern __shared__ __align__(1024) uint8_t shared[];
    const bool loads = (int)threadIdx.x >= 128 * C::kTeams;
    const int team = __shfl_sync(0xffffffffu, loads ? (int)threadIdx.x / 32 - kWarps * C::kTeams : (int)threadIdx.x / 128, 0);      // (the fourth loading warp: none)
    uint8_t *smem = shared + min(team, C::kTeams - 1) * C::kTeam;
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + C::offBar), *empty = full + S;
    volatile uint32_t *live = reinterpret_cast<uint32_t *>(empty + S), *abortp = live + S;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32 % kWarps, 0), lane = tid % 32;
    if (!loads && tid % 128 == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full + s, 1); mbar_init(empty + s, kWarps); }
        *abortp = 0;
        fence_mbar_init();
    }
    // (unless a cluster does a whole head, the kernel in front is the one that clears the counters: only who uses them waits for it)
    if (kClusters && a.nc == 1) {
        grid_dependency_wait();
        grid_launch_dependents();
    }
    const int *lens = after_wait(a.lens), *table = after_wait(a.table);
    if constexpr (kClusters) __syncthreads();                    // (else the barriers of find_share are those of the set-up too)
    const Share sh = kClusters ? cluster_share<C>(a, lens, min(team, C::kTeams - 1))
                              : find_share<C>(a, lens, reinterpret_cast<int *>(shared + C::offScan), min(team, C::kTeams - 1));
    const int count = sh.u1 - sh.u0;
    Place<C> at{};
    if (count > 0 || kClusters) {
        const int len = length_of(a, lens, sh.b), end = units_of<C::kUnitKeys>(len), in = sh.u0 - sh.before;
        at.set(sh.b, in / end, in % end, len);
    }

    if (loads) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLoadRegs));
        if (team < C::kTeams && count > 0) {
        // ------------------------------------------------------------------ loads: a lane per block, four units to a batch of table entries
            constexpr int kBatch = 32 / C::kBlocks;
            const uint8_t *pool = after_wait(a.pool);
            const int mine = lane / C::kBlocks, block = lane % C::kBlocks;
            ArmCounts<S> armed;
            int base = at.t, nb, nh, nlen, stage = 0, round = 0;
            long long cur = block_offset<D, true, C>(a, table, at.b, at.h, base + mine, block), nxt;
            auto fetch_next = [&] {      // the batch behind the current one
                nb = at.b; nh = at.h; nlen = at.len;
                int nt = base + kBatch;
                if (nt >= at.end) {
                    nt = 0;
                    if (++nh == a.Hkv) { nh = 0; nlen = length_of(a, lens, ++nb); }
                }
                nxt = block_offset<D, true, C>(a, table, nb, nh, nt + mine, block);
            };
            fetch_next();
            for (int i = 0; i < count; ++i) {
                bool ok = round == 0 || mbar_wait(empty + stage, (round - 1) & 1, abortp, a.status, PERR_EMPTY);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const bool valid = mine == at.t - base && cur >= 0 && at.t * C::kUnitKeys + 16 * block < at.len;
                const uint32_t who = __ballot_sync(0xffffffffu, valid);
                if (lane == 0) {
                    live[stage] = who >> ((at.t - base) * C::kBlocks);
                    mbar_arm(full, stage, (uint32_t)(__popc(who) * C::kBlock), armed);
                }
                __syncwarp();
                if (valid) bulk_load_1d(smem + stage * kUnit + block * C::kBlock, pool + cur, C::kBlock, full + stage);
                if (++stage == S) { stage = 0; ++round; }
                ++at.t;
                const bool over = at.t == at.end;
                if (over || at.t == base + kBatch) {
                    if (over) at.set(nb, nh, 0, nlen);
                    base = at.t;
                    cur = nxt;
                    fetch_next();
                }
            }
            if (lane == 0) mbar_drain(full, armed);      // copies still on their way land before the CTA leaves (bounded)
        }
        __syncwarp();
        if constexpr (kClusters) finish_clusters<D, true, NQ>(a, shared, reinterpret_cast<unsigned int *>(shared + C::offFlag), -1, 128 * C::kTeams);
        return;
    }

    // ---------------------------------------------------------------------- use
    const float scale = a.scale_log2 * exp2i(-kCodeExp1 - kLift), margin = kRescale / scale;
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kUseRegs));
    if (!kClusters || a.nc > 1) {
        grid_dependency_wait();
        grid_launch_dependents();
    }
    const uint32_t ring = smem_u32(smem);
    int stage = 0, parity = 0;
    bool ok = true;
    walk<D, true, NQ, kClusters>(a, sh, at, after_wait(a.q), lens, smem, team, [&](HeadState<D, true, NQ> &s, const Place<C> &use) {
        if (ok && !mbar_wait(full + stage, parity, abortp, a.status, PERR_FULL)) ok = false;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        const uint32_t here = live[stage] >> (C::kSub * warp) & ((1u << C::kSub) - 1);
        if (here) s.step(ring + stage * kUnit + warp * C::kSub * C::kBlock, here, use.len - (use.t * C::kUnitKeys + 16 * C::kSub * warp), scale, margin, lane);
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + stage);
        if (++stage == S) { stage = 0; parity ^= 1; }
    });
    if constexpr (kClusters) {
        __syncwarp();
        finish_clusters<D, true, NQ>(a, shared, reinterpret_cast<unsigned int *>(shared + C::offFlag), tid, 128 * C::kTeams);
    }
}

template <int D, int NQ, bool kClusters>
__global__ void __launch_bounds__((Cfg<D, false, NQ>::kThreads), (Cfg<D, false, NQ>::kCtas)) paged_decode16_kernel(const PagedArgs a)
{
    using C = Cfg<D, false, NQ>;
    constexpr int S = C::kStages;
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32;
    // (unless a cluster does a whole head, the kernel in front is the one that clears the counters: only who uses them waits for it)
    if (kClusters && a.nc == 1) {
        grid_dependency_wait();
        grid_launch_dependents();
    }
    const int *lens = after_wait(a.lens), *table = after_wait(a.table);
    const uint8_t *pool = after_wait(a.pool);
    const Share sh = kClusters ? cluster_share<C>(a, lens, 0) : find_share<C>(a, lens, reinterpret_cast<int *>(smem + C::offScan), 0);
    const int count = sh.u1 - sh.u0;
    if (count == 0 && !kClusters) return;
    Place<C> ask;
    {
        const int len = length_of(a, lens, sh.b), end = units_of<C::kUnitKeys>(len), in = sh.u0 - sh.before;
        ask.set(sh.b, in / end, in % end, len);
    }
    const Place<C> start = ask;

    // ---- requests: S - 1 steps ahead of their use
    const uint32_t ring = smem_u32(smem) + warp * S * C::kBlock;
    int left_to_ask = count, base = ask.t, nb, nh, nlen;      // base: unit of the batch's first entry
    uint32_t live = 0;                                        // stages that hold keys
    long long cur = block_offset<D, false, C>(a, table, ask.b, ask.h, base + lane, warp), nxt;
    auto fetch_next = [&] {      // the batch behind the current one
        nb = ask.b; nh = ask.h; nlen = ask.len;
        int nt = base + 32;
        if (nt >= ask.end) {
            nt = 0;
            if (++nh == a.Hkv) { nh = 0; nlen = length_of(a, lens, ++nb); }
        }
        nxt = block_offset<D, false, C>(a, table, nb, nh, nt + lane, warp);
    };
    fetch_next();
    auto request = [&](int stage) {
        live &= ~(1u << stage);
        if (left_to_ask > 0) {
            --left_to_ask;
            const long long at = __shfl_sync(0xffffffffu, cur, ask.t - base);
            const int left = ask.len - (ask.t * C::kUnitKeys + 16 * warp);
            if (at >= 0 && left > 0) {
                // rows past the end of the sequence are filled with zeros: whatever they hold, their weight is 0
                constexpr int kRow = D / 8, kAt = 32 / kRow;
                const int c = lane % kRow;
                live |= 1u << stage;
#pragma unroll
                for (int i = 0; i < 16 / kAt; ++i) {
                    const int r = i * kAt + lane / kRow, bytes = r < left ? 16 : 0;
                    const uint32_t to = ring + stage * C::kBlock + r * (2 * D) + ((c & ~7) | ((c ^ r) & 7)) * 16;
                    const uint8_t *from = pool + at + (bytes ? r * (2 * D) + c * 16 : 0);
                    cp_async16(to, from, bytes);
                    cp_async16(to + 32 * D, from + (long long)a.page * (2 * D), bytes);
                }
            }
            ++ask.t;
            const bool over = ask.t == ask.end;
            if (over || ask.t == base + 32) {
                if (over) ask.set(nb, nh, 0, nlen);
                base = ask.t;
                cur = nxt;
                fetch_next();
            }
        }
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i) request(i);

    // ---- use
    if (!kClusters || a.nc > 1) {
        grid_dependency_wait();
        grid_launch_dependents();
    }
    const float margin = kRescale / a.scale_log2;
    int get = 0;      // stage of this step
    walk<D, false, NQ, kClusters>(a, sh, start, after_wait(a.q), lens, smem, 0, [&](HeadState<D, false, NQ> &s, const Place<C> &use) {
        cp_wait<S - 2>();
        __syncwarp();
        const uint32_t st = ring + get * C::kBlock, here = live >> get & 1;
        request(get == 0 ? S - 1 : get - 1);      // (into the stage of the step before)
        get = get == S - 1 ? 0 : get + 1;
        if (here) s.step(st, here, use.len - (use.t * C::kUnitKeys + 16 * warp), a.scale_log2, margin, lane);
    });
    if constexpr (kClusters) {
        __syncwarp();
        finish_clusters<D, false, NQ>(a, smem, reinterpret_cast<unsigned int *>(smem + C::offFlag), tid, 128);
    } else {
        cp_wait<0>();
    }
}

int shares_for(const PagedProblem &p, int per_sm, int unit)
{
    // (a unit for a share at least, at the lengths that the table has room for)
    const long long units = (long long)p.B * p.pool.Hkv * (((long long)p.max_pages * p.pool.page + unit - 1) / unit), most = (long long)per_sm * device_info().sms;
    return (int)(units < most ? units : most);
}

template <int D, bool kInt4, int NQ>
cudaError_t launch(const PagedProblem &p, const void *q, const void *pool, const int *table, const int *lens, void *out, float *lse, void *ws,
                   cudaStream_t st)
{
    using C = Cfg<D, kInt4, NQ>;
    constexpr auto kernel = [] { if constexpr (kInt4) return paged_decode4_kernel<D, NQ, false>; else return paged_decode16_kernel<D, NQ, false>; }();
    constexpr auto clusters = [] { if constexpr (kInt4) return paged_decode4_kernel<D, NQ, true>; else return paged_decode16_kernel<D, NQ, true>; }();
    const int G = p.H / p.pool.Hkv, sms = device_info().sms, shares = shares_for(p, C::kShares, C::kUnitKeys), most = 4 * sms;
    // Equal shares of everything, or one or more clusters for each head: by the time that each takes in nanoseconds, for the lengths that the tables have room
    // for.  HBM gives 6500 bytes in one; an SM takes 60, of 4-bit blocks 38 (it computes for longer).  One cluster for a head needs no counters
    // and no second join; shares of few heads are many parts, which one team joins, 128 elements at once and four parts on their way.  Clusters of 4 and 8
    // leave SMs of a GPC over.  (B8 H8/8 n8192 d128 bf16: clusters of four 43 us, shares 48; B1 H8/1 n131072 4 bits: 15 clusters of eight 15 us, one
    // cluster 60, shares 92; B64 H32/8 of 4000 keys 4 bits: shares 78, clusters do not fit.)
    const int heads = p.B * p.pool.Hkv, slots = C::kCtas * sms, units = (int)(((long long)p.max_pages * p.pool.page + C::kUnitKeys - 1) / C::kUnitKeys);
    constexpr double kUnitBytes = (double)C::kBlocks * C::kBlock, kSmRate = kInt4 ? 38.0 : 60.0;
    const double hbm = kUnitBytes * units * heads / 6500.0;
    auto stream = [&](double units_of_a_team, double teams_on_an_sm) { return std::max(hbm, std::ceil(units_of_a_team) * kUnitBytes * teams_on_an_sm / kSmRate); };
    const double equal = std::max(1.0, (double)units * heads / (C::kShares * sms)), parts = std::min((double)units, std::max(1.0, (double)C::kShares * sms / heads));
    double best = stream(equal, C::kShares) + 2500.0 + 700.0 * std::ceil(parts / 4.0) * ((G * (D / 4) + 127) / 128);
    int cl = 0, nc = 0;
    for (int c = 1; c <= 8; c *= 2) {
        const long long at_once = slots * (c == 8 ? 85LL : c == 4 ? 90LL : 100LL) / (100LL * c);
        if (heads > at_once) break;
        const int most = (int)std::min<long long>(at_once / heads, (units + c * C::kTeams - 1) / (c * C::kTeams));
        for (int n : {1, most}) {
            const double cost = stream((double)units / (n * c * C::kTeams), (double)((heads * n * c + sms - 1) / sms) * C::kTeams) + (n > 1 ? 5000.0 : 1500.0);
            if (cost < best || (cost == best && cl)) { best = cost; cl = c; nc = n; }
        }
    }
    const int ctas = cl ? heads * nc * cl : std::min(shares, slots);
    PagedArgs a{};
    a.q = (const __nv_bfloat16 *)q; a.pool = (const uint8_t *)pool; a.table = table; a.lens = lens;
    a.out = (__nv_bfloat16 *)out; a.lse = lse;
    a.part_o = (float *)ws;
    a.part_ml = a.part_o + (size_t)2 * most * G * D;
    a.counters = (unsigned int *)(a.part_ml + (size_t)2 * most * G * 2);
    a.sq = p.sq;
    a.table_stride = p.table_stride; a.page_stride = p.pool.page_stride;
    a.B = p.B; a.Hkv = p.pool.Hkv; a.G = G; a.pages = p.pool.pages; a.page = p.pool.page;
    a.cap = (int)((long long)p.max_pages * p.pool.page);
    a.by_page = FastDiv((uint32_t)p.pool.page);
    a.status = device_status_ptr();
    a.cl = cl;
    a.nc = nc;
    a.scale_log2 = p.scale == 0.f ? 1.f : fabsf(p.scale) * kLog2e;
    a.sign2 = p.scale == 0.f ? 0u : p.scale > 0.f ? 0x3f803f80u : 0xbf80bf80u;
    cudaError_t e = cl ? allow_smem<clusters>(C::kTotal) : allow_smem<kernel>(C::kTotal);
    if (e == cudaSuccess && (!cl || nc > 1)) e = decode_clear(a.counters, most, st);
    if (e != cudaSuccess) return e;
    LaunchScope scope(MOA_KERNEL_OTHER, st);
    const dim3 grid((unsigned)ctas), block(C::kThreads);
    return cl ? launch_cluster(clusters, (unsigned)cl, grid, block, (size_t)C::kTotal, st, a)
              : launch_dependent(kernel, grid, block, (size_t)C::kTotal, st, a);
}

}  // namespace

size_t paged_decode_workspace_bytes(const PagedProblem &p)
{
    const size_t most = (size_t)4 * device_info().sms, G = (size_t)(p.H / p.pool.Hkv);
    return 2 * most * G * (p.pool.d + 2) * sizeof(float) + most * sizeof(unsigned int);
}

cudaError_t paged_decode(const PagedProblem &p, const void *q, const void *pool, const int *table, const int *lens, void *out, float *lse,
                         void *ws, cudaStream_t st)
{
    const bool two = p.H / p.pool.Hkv > 8;
    if (p.pool.d == 64) {
        if (p.pool.int4) return two ? launch<64, true, 2>(p, q, pool, table, lens, out, lse, ws, st) : launch<64, true, 1>(p, q, pool, table, lens, out, lse, ws, st);
        return two ? launch<64, false, 2>(p, q, pool, table, lens, out, lse, ws, st) : launch<64, false, 1>(p, q, pool, table, lens, out, lse, ws, st);
    }
    if (p.pool.int4) return two ? launch<128, true, 2>(p, q, pool, table, lens, out, lse, ws, st) : launch<128, true, 1>(p, q, pool, table, lens, out, lse, ws, st);
    return two ? launch<128, false, 2>(p, q, pool, table, lens, out, lse, ws, st) : launch<128, false, 1>(p, q, pool, table, lens, out, lse, ws, st);
}

}  // namespace moa
