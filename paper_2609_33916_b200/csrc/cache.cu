// The paged cache's append (rotation, rounding or quantisation, and the writes into the pages in one launch) and its read-back.
//
// HBM-bound: q is read and written once, k and v are read once and written as 2 or 0.5625 bytes per element.  As in rope.cu a block takes a few
// tokens with all their rows (queries, keys, values), the angles of a token are made once and shared through shared memory, and a row is d / 16
// lanes with two 16-byte pieces each, several rows in flight per lane.
//
// K is rounded to the nearest bf16 of the exact rotation, subnormal ones included.  In 32 bits the rotation is within 4.5 * 2^-24 f (|x1| + |x2|) of it (cosine
// and sine 1.5, the factor, a product and the sum one each), and 2^-147; where the two ends of that interval round apart, one element in about 5000, it is made again in 64 bits.
// So what a key quantises to does not depend on which arithmetic turned it, and a 4-bit page is a function of the bf16 page's bits.
//
// Quantising: 32 neighbours share a scale s = bf16(amax / 7); x / s with one correction by the remainder is exact wherever the quotient is a tie
// between two codes (x has 8 bits, the code and a half 4), so that halves go to even as the definition says.
#include "cache_layout.cuh"

namespace moa {
namespace {

using namespace ptx;

constexpr int kThreads = 128, kTokens = 2, kUnroll = 2, kResident = 8;
using Piece = Chunk<__nv_bfloat16, 8>;

// x / d where x may pass 31 bits
__device__ __forceinline__ long long divide(long long x, const FastDiv &by) { return x < (1LL << 31) ? (long long)by.div((uint32_t)x) : x / by.d; }

struct AppendArgs {
    const __nv_bfloat16 *q, *k, *v;
    const int *pos;
    const long long *slot;
    const float *inv_freq;
    __nv_bfloat16 *qo;
    uint8_t *pool;
    RopeStride sq, sk, sv, so;
    long long page_stride, keys;     // keys: of the whole pool
    int T, H, Hkv, page, d_rot, tt;
    FastDiv by_heads, by_kv, by_page, by_freqs;      // H, H_kv, page, d_rot / 2
    float factor;
};

// The nearest bf16 of a double, in one rounding: half to even on the 45 bits that go, or, where bf16 is subnormal, by a sum whose last place is its step.
__device__ __forceinline__ float round_bf16(double v)
{
    const double a = fabs(v);
    if (a < 0x1p-126) return (float)copysign((a + 0x1.8p-81) - 0x1.8p-81, v);
    if (!(a < INFINITY)) return (float)v;
    long long b = __double_as_longlong(v);
    b = (b + ((1LL << 44) - 1) + ((b >> 45) & 1)) & ~((1LL << 45) - 1);
    return (float)__longlong_as_double(b);      // (2^128 and above: infinity)
}

// A rotated pair, f (x1 cos - x2 sin) and f (x2 cos + x1 sin), in 64 bits and rounded to bf16.
__device__ __noinline__ float2 exact_turn(float x1, float x2, int pos, float f, float factor)
{
    double s, c;
    sincospi(2.0 * part_of_turn(pos, f), &s, &c);
    c *= (double)factor;
    s *= (double)factor;
    return make_float2(round_bf16((double)x1 * c - (double)x2 * s), round_bf16((double)x2 * c + (double)x1 * s));
}

// Element i of eight, by selects (i is known at run time only)
__device__ __forceinline__ uint32_t bf16_at(const uint4 &w, int i)
{
    const uint32_t v = i < 4 ? (i < 2 ? w.x : w.y) : (i < 6 ? w.z : w.w);
    return i & 1 ? v >> 16 : v & 0xffffu;
}
__device__ __forceinline__ void put_bf16(uint4 &w, int i, uint32_t bits)
{
    const uint32_t keep = i & 1 ? 0xffffu : 0xffff0000u, put = i & 1 ? bits << 16 : bits;
    if (i / 2 == 0) w.x = (w.x & keep) | put;
    if (i / 2 == 1) w.y = (w.y & keep) | put;
    if (i / 2 == 2) w.z = (w.z & keep) | put;
    if (i / 2 == 3) w.w = (w.w & keep) | put;
}

// Of 16 elements of a lane (the lanes of a pair hold a group): codes of 1..15, four bits each in the order of the elements (the first lowest),
// and the group's scale.
__device__ __forceinline__ void quantise16(const Piece &lo, const Piece &hi, uint32_t (&code)[2], uint16_t &scale)
{
    float x[2][8];
    lo.unpack(x[0]);
    hi.unpack(x[1]);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, max(__float_as_uint(x[0][i]) & 0x7fffffffu, __float_as_uint(x[1][i]) & 0x7fffffffu));      // (NaN is the largest)
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    const float amax = __uint_as_float(most);
    float s = __bfloat162float(__float2bfloat16_rn(amax / 7.f));
    const bool plain = most < 0x7f800000u && amax >= 0x1p-100f;
    s = plain ? s : most >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : 0.f;
    const float inv = plain ? 1.f / s : 0.f;
    code[0] = code[1] = 0x88888888u;
    if (plain) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            // Adding 1.5 * 2^23 + 8 leaves the code, rounded half to even, in the low bits (|x / s| <= 7 (1 + 2^-8): at most 7); the words of all eight,
            // each 16 times the next, add up to the codes and a constant.
            uint32_t c = 0;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const float v = x[w][i], q0 = v * inv, q1 = fmaf(fmaf(-q0, s, v), inv, q0);
                c = c * 16u + __float_as_uint(q1 + 12582920.f);
            }
            code[w] = c - 0x4b400000u * 0x11111111u;
        }
    }
    scale = (uint16_t)(__float_as_uint(s) >> 16);
}

// Nibbles 0..7 (elements 8 t .. 8 t + 7 of a group) in the order of a word of K codes: the even elements, then the odd ones
__device__ __forceinline__ uint32_t even_then_odd(uint32_t c)
{
    uint32_t e = c & 0x0f0f0f0fu, o = (c >> 4) & 0x0f0f0f0fu;
    e = (e | (e >> 4)) & 0x00ff00ffu;
    o = (o | (o >> 4)) & 0x00ff00ffu;
    e = (e | (e >> 8)) & 0xffffu;
    o = (o | (o >> 8)) & 0xffffu;
    return e | (o << 16);
}

// Where the codes and the scale of a lane's 16 elements (group y0, half `half` of it) go
template <int D>
__device__ __forceinline__ void write_k4(uint8_t *blk, int r, int y0, int half, const uint32_t (&code)[2], uint16_t scale)
{
    using L = Block4<D>;
    *reinterpret_cast<uint32_t *>(blk + L::k_word(r, 2 * half, y0)) = even_then_odd(code[0]);
    *reinterpret_cast<uint32_t *>(blk + L::k_word(r, 2 * half + 1, y0)) = even_then_odd(code[1]);
    if (half == 0) *reinterpret_cast<uint16_t *>(blk + L::k_scale(r, y0)) = scale;
}
// V: a word holds four elements of two neighbouring groups: the lanes of those have traded halves of their codes
template <int D>
__device__ __forceinline__ void write_v4(uint8_t *blk, int r, int y0, int half, const uint32_t (&code)[2], uint32_t trade, uint16_t scale)
{
    using L = Block4<D>;
    const uint32_t mine = code[y0 % 2 ? 1 : 0], even = y0 % 2 ? trade : mine, odd = y0 % 2 ? mine : trade;
    const int g = 4 * half + (y0 % 2 ? 2 : 0);
    *reinterpret_cast<uint32_t *>(blk + L::v_word(r, g, y0 / 2)) = (even & 0xffffu) | (odd << 16);
    *reinterpret_cast<uint32_t *>(blk + L::v_word(r, g + 1, y0 / 2)) = (even >> 16) | (odd & 0xffff0000u);
    if (half == 0) *reinterpret_cast<uint16_t *>(blk + L::v_scale(r, y0)) = scale;
}

// The pieces of a key turned and rounded to the nearest bf16 of the exact result.  pos, f: of this lane's pairs
template <bool kPairs>
__device__ __forceinline__ void turn_key(Piece &x, Piece &y, const float (&c)[8], const float (&s)[8], float factor, const int *pos, const float *f)
{
    float fx[8], fy[8], e[8];
    const uint4 xi = x.w, yi = y.w;
    x.unpack(fx);
    y.unpack(fy);
    const float f1 = fmaxf(fabsf(factor), 0x1p-100f);      // (below, the factor's products are not within 2^-24)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x1 = kPairs ? (i < 4 ? fx[2 * i] : fy[2 * i - 8]) : fx[i], x2 = kPairs ? (i < 4 ? fx[2 * i + 1] : fy[2 * i - 7]) : fy[i];
        // (what a part of the rotation may overflow with, this product does: then the pair is in doubt.  Where results are subnormal, each of three
        // roundings is off by 2^-150 whatever the size: 2^-147, unless both elements are 0)
        const float size = f1 * (fabsf(x1) + fabsf(x2));
        e[i] = fmaxf(2.8e-7f * size, fminf(size, 0x1p-147f));
    }
    rotate<8, kPairs>(fx, fy, c, s);
    uint32_t doubt = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y1 = kPairs ? (i < 4 ? fx[2 * i] : fy[2 * i - 8]) : fx[i], y2 = kPairs ? (i < 4 ? fx[2 * i + 1] : fy[2 * i - 7]) : fy[i];
        if (pack_bf16(y1 - e[i], y2 - e[i]) != pack_bf16(y1 + e[i], y2 + e[i])) doubt |= 1u << i;
    }
    x.pack(fx);
    y.pack(fy);
    while (doubt) {
        const int i = __ffs((int)doubt) - 1;
        doubt &= doubt - 1;
        const int at1 = kPairs ? 2 * i & 7 : i, at2 = kPairs ? at1 + 1 : i;
        const bool first = !kPairs || i < 4;      // (pairs: in the first piece or in the second)
        const uint32_t b1 = bf16_at(first ? xi : yi, at1), b2 = bf16_at(kPairs && first ? xi : yi, at2);
        const float2 z = exact_turn(__uint_as_float(b1 << 16), __uint_as_float(b2 << 16), *pos, f[i], factor);
        const uint32_t z1 = __float_as_uint(z.x) >> 16, z2 = __float_as_uint(z.y) >> 16;
        if (first) put_bf16(x.w, at1, z1); else put_bf16(y.w, at1, z1);
        if (kPairs && first) put_bf16(x.w, at2, z2); else put_bf16(y.w, at2, z2);
    }
}

// Blocks of a tile of tokens: gridDim.y == 1: one with all its rows; else the first one keys and values (they take longest: 64 tokens 8.4 us with them in the
// last one, 7.9 in the first), the others the queries
template <int D, bool kInt4, bool kPairs>
__global__ void __launch_bounds__(kThreads, kResident) kv_append_kernel(const AppendArgs a)
{
    constexpr int kLanes = D / 16, kPer = kThreads / kLanes;
    __shared__ float4 angles[kTokens * D / 4];
    const int tid = threadIdx.x, lane = tid % 32, t0 = blockIdx.x * a.tt, nt = min(a.tt, a.T - t0), freqs = a.d_rot / 2, np = a.d_rot / 16;
    grid_dependency_wait();
    grid_launch_dependents();
    const int *pos = after_wait(a.pos);
    const float *inv_freq = after_wait(a.inv_freq);
    const long long *slots = after_wait(a.slot);
    const __nv_bfloat16 *q = after_wait(a.q), *k = after_wait(a.k), *v = after_wait(a.v);
    const int r0 = tid / kLanes, p = tid % kLanes;
    const bool turns = p < np;
    const int c0 = turns && !kPairs ? 8 * p : 16 * p, c1 = turns && !kPairs ? freqs + 8 * p : c0 + 8;      // elements, for q and k; v: 16 p and 16 p + 8
    const int qparts = gridDim.y == 1 ? 1 : (int)gridDim.y - 1, qpart = gridDim.y == 1 ? 0 : blockIdx.y == 0 ? qparts : (int)blockIdx.y - 1;
    const bool kv = gridDim.y == 1 || qpart == qparts;
    const int qrows = qpart < qparts ? nt * a.H : 0, kvrows = kv ? nt * a.Hkv : 0;
    // the first rows are on their way while the angles are made
    Piece x[kUnroll], y[kUnroll];
    int tok[kUnroll], head[kUnroll];
    auto load_q = [&](int row) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u, row += kPer) {
            tok[u] = -1;
            if (row >= qrows) continue;
            tok[u] = (int)a.by_heads.div((uint32_t)row);
            head[u] = row - tok[u] * a.H;
            const __nv_bfloat16 *src = q + a.sq.at(t0 + tok[u], head[u]);
            x[u].w = *reinterpret_cast<const uint4 *>(src + c0);
            y[u].w = *reinterpret_cast<const uint4 *>(src + c1);
        }
    };
    int row = qpart * (kPer * kUnroll) + r0;
    load_q(row);
    for (int i = tid; i < nt * freqs; i += kThreads) {
        const int t = (int)a.by_freqs.div((uint32_t)i), f = i - t * freqs;
        float2 cs = position_angle(pos[t0 + t], inv_freq[f]);
        cs.x *= a.factor;
        cs.y *= a.factor;
        write_angle<8>(angles + t * (freqs / 2), np, f, cs);
    }
    __syncthreads();
    while (row < qrows) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (tok[u] < 0) continue;
            if (turns) {
                float fx[8], fy[8], c[8], s[8];
                x[u].unpack(fx);
                y[u].unpack(fy);
                read_angles<8>(angles + tok[u] * (freqs / 2), np, p, c, s);
                rotate<8, kPairs>(fx, fy, c, s);
                x[u].pack(fx);
                y[u].pack(fy);
            }
            __nv_bfloat16 *dst = a.qo + a.so.at(t0 + tok[u], head[u]);
            *reinterpret_cast<uint4 *>(dst + c0) = x[u].w;
            *reinterpret_cast<uint4 *>(dst + c1) = y[u].w;
        }
        row += qparts * (kPer * kUnroll);
        load_q(row);
    }
    // keys and values: a lane has the pieces of both of a head.  (All lanes of a warp make the same rounds: the exchanges are of whole warps.)
    for (int base = 0; base < kvrows; base += kPer) {
        const int r = base + r0;
        const bool in = r < kvrows;
        const int t = in ? (int)a.by_kv.div((uint32_t)r) : 0, h = in ? r - t * a.Hkv : 0;
        const __nv_bfloat16 *ks = k + a.sk.at(t0 + t, h), *vs = v + a.sv.at(t0 + t, h);
        Piece kx, ky, vx, vy;
        kx.w = *reinterpret_cast<const uint4 *>(ks + c0);
        ky.w = *reinterpret_cast<const uint4 *>(ks + c1);
        vx.w = *reinterpret_cast<const uint4 *>(vs + 16 * p);
        vy.w = *reinterpret_cast<const uint4 *>(vs + 16 * p + 8);
        const long long at = slots[t0 + t];
        const bool there = in && at >= 0 && at < a.keys;
        const long long pg = there ? divide(at, a.by_page) : 0;
        const int key = there ? (int)(at - pg * a.page) : 0;
        uint8_t *page = a.pool + pg * a.page_stride;
        if (turns) {
            float c[8], s[8];
            read_angles<8>(angles + t * (freqs / 2), np, p, c, s);
            turn_key<kPairs>(kx, ky, c, s, a.factor, pos + t0 + t, inv_freq + 8 * p);
        }
        if constexpr (!kInt4) {
            if (there) {
                uint8_t *dst = page + row16(a.page, D, h, 0, key), *dv = dst + (long long)a.page * (2 * D);
                *reinterpret_cast<uint4 *>(dst + 2 * c0) = kx.w;
                *reinterpret_cast<uint4 *>(dst + 2 * c1) = ky.w;
                *reinterpret_cast<uint4 *>(dv + 32 * p) = vx.w;
                *reinterpret_cast<uint4 *>(dv + 32 * p + 16) = vy.w;
            }
        } else {
            // the half layout's lanes hold pieces p and p + d_rot / 16: each gets pieces 2 p and 2 p + 1 from the lanes that have them
            if (!kPairs && np > 0) {
                uint4 got[2];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const int piece = 2 * p + w;
                    const bool second = piece >= np && turns;
                    const int from = lane - p + (turns ? (second ? piece - np : piece) : p);
                    got[w].x = __shfl_sync(0xffffffffu, kx.w.x, from);
                    got[w].y = __shfl_sync(0xffffffffu, kx.w.y, from);
                    got[w].z = __shfl_sync(0xffffffffu, kx.w.z, from);
                    got[w].w = __shfl_sync(0xffffffffu, kx.w.w, from);
                    const uint32_t y0 = __shfl_sync(0xffffffffu, ky.w.x, from), y1 = __shfl_sync(0xffffffffu, ky.w.y, from);
                    const uint32_t y2 = __shfl_sync(0xffffffffu, ky.w.z, from), y3 = __shfl_sync(0xffffffffu, ky.w.w, from);
                    if (second) got[w] = make_uint4(y0, y1, y2, y3);
                }
                if (turns) { kx.w = got[0]; ky.w = got[1]; }
            }
            const int y0 = p / 2, half = p % 2, rk = key % kBlockKeys;      // group, and which 16 of it
            uint8_t *blk = page + block4<D>(a.page, h, key / kBlockKeys);
            uint32_t code[2];
            uint16_t scale;
            quantise16(kx, ky, code, scale);
            if (there) write_k4<D>(blk, rk, y0, half, code, scale);
            quantise16(vx, vy, code, scale);
            const uint32_t trade = __shfl_xor_sync(0xffffffffu, code[y0 % 2 ? 0 : 1], 2);
            if (there) write_v4<D>(blk, rk, y0, half, code, trade, scale);
        }
    }
}

struct GatherArgs {
    const uint8_t *pool;
    const long long *slot;
    void *k, *v;
    RopeStride sk, sv;
    long long page_stride, keys;           // keys: of the whole pool
    int T, Hkv, page;
    FastDiv by_page;
};

// Four codes, nibbles 0..3 of the low half of h in the order of the elements, or eight of K's word, as pairs at the low ends of the halves of a word
__device__ __forceinline__ void spread(uint32_t h, uint32_t (&pair)[2])
{
    pair[0] = (h | h << 12) & 0x000f000fu;
    pair[1] = (h >> 8 | h << 4) & 0x000f000fu;
}
// Pairs of codes to values: 128 + c as bf16, minus 136, times the scale: exact until the product's one rounding
__device__ __forceinline__ void store_codes(__nv_bfloat16 *p, const uint32_t (&pair)[4], uint32_t scale)
{
    uint32_t w[4];
    const uint32_t s2 = scale | scale << 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = pair[i] | 0x43004300u;
        asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(w[i]) : "r"(x), "r"(0xc308c308u));
        asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(s2));
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_codes(float *p, const uint32_t (&pair)[4], uint32_t scale)
{
    const float s = __uint_as_float(scale << 16);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = s * (float)((int)(pair[i] & 15u) - 8);
        f[2 * i + 1] = s * (float)((int)(pair[i] >> 16) - 8);
    }
    reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store16(__nv_bfloat16 *p, const uint4 &w) { *reinterpret_cast<uint4 *>(p) = w; }
__device__ __forceinline__ void store16(float *p, const uint4 &w)
{
    Piece x;
    float f[8];
    x.w = w;
    x.unpack(f);
    reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// A row of a head is d / 8 lanes with 8 elements each.  A block takes 16 tokens (the codes of 16 neighbouring values share sectors) and kGatherRows
// heads of K or of V: first the slots, then all codes and scales of a lane are on their way, then the results.
constexpr int kGatherRows = 4, kGatherTokens = 16;

template <typename T, int D, bool kInt4, bool kV>
__device__ __forceinline__ void gather_rows(const GatherArgs &a, const uint8_t *pool, long long at, int t, int h0)
{
    using L = Block4<D>;
    const int c = threadIdx.x % (D / 8), y = c / 4, t8 = c % 4;
    const bool there = at >= 0 && at < a.keys;
    const long long pg = there ? divide(at, a.by_page) : 0;
    const int key = there ? (int)(at - pg * a.page) : 0, r = key % kBlockKeys;
    const uint8_t *page = pool + pg * a.page_stride;
    uint4 raw[kGatherRows];        // 16 bytes of a row; 4 bits: one or two words of codes, and the scale
#pragma unroll
    for (int u = 0; u < kGatherRows; ++u) {
        raw[u] = make_uint4(0u, 0u, 0u, 0u);
        if (!there || h0 + u >= a.Hkv) continue;
        if constexpr (!kInt4) {
            raw[u] = *reinterpret_cast<const uint4 *>(page + row16(a.page, D, h0 + u, kV, key) + 16 * c);
        } else {
            const uint8_t *blk = page + block4<D>(a.page, h0 + u, key / kBlockKeys);
            raw[u].x = *reinterpret_cast<const uint32_t *>(blk + (kV ? L::v_word(r, 2 * t8, y / 2) : L::k_word(r, t8, y)));
            if (kV) raw[u].y = *reinterpret_cast<const uint32_t *>(blk + L::v_word(r, 2 * t8 + 1, y / 2));
            raw[u].z = *reinterpret_cast<const uint16_t *>(blk + (kV ? L::v_scale(r, y) : L::k_scale(r, y)));
        }
    }
    T *dst = kV ? (T *)a.v + a.sv.at(t, h0) : (T *)a.k + a.sk.at(t, h0);
    const int step = kV ? a.sv.head : a.sk.head;
#pragma unroll
    for (int u = 0; u < kGatherRows; ++u) {
        if (h0 + u >= a.Hkv) break;
        T *p = dst + (long long)u * step + 8 * c;
        if constexpr (!kInt4) {
            store16(p, raw[u]);
        } else {
            uint32_t pair[4];      // (no such slot: scale 0)
            if (kV) {
                const int sh = 16 * (y % 2);
                uint32_t lo[2], hi[2];
                spread((raw[u].x >> sh) & 0xffffu, lo);
                spread((raw[u].y >> sh) & 0xffffu, hi);
                pair[0] = lo[0]; pair[1] = lo[1]; pair[2] = hi[0]; pair[3] = hi[1];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) pair[i] = raw[u].x >> (4 * i) & 0x000f000fu;
            }
            if (!there) pair[0] = pair[1] = pair[2] = pair[3] = 0x00080008u;      // (+0)
            store_codes(p, pair, raw[u].z);
        }
    }
}

template <typename T, int D, bool kInt4>
__global__ void __launch_bounds__(kGatherTokens * D / 8) kv_gather_kernel(const GatherArgs a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const uint8_t *pool = after_wait(a.pool);
    const long long *slots = after_wait(a.slot);
    const int t = blockIdx.x * kGatherTokens + threadIdx.x / (D / 8), parts = (int)gridDim.y / 2, part = (int)blockIdx.y;
    if (t >= a.T) return;
    const long long at = slots[t];
    if (part < parts)
        gather_rows<T, D, kInt4, false>(a, pool, at, t, part * kGatherRows);
    else
        gather_rows<T, D, kInt4, true>(a, pool, at, t, (part - parts) * kGatherRows);
}

template <int D, bool kInt4>
cudaError_t launch_append(const AppendArgs &a, bool pairs, dim3 grid, cudaStream_t st)
{
    LaunchScope scope(MOA_KERNEL_OTHER, st);
    return pairs ? launch_dependent(kv_append_kernel<D, kInt4, true>, grid, dim3(kThreads), (size_t)0, st, a)
                 : launch_dependent(kv_append_kernel<D, kInt4, false>, grid, dim3(kThreads), (size_t)0, st, a);
}

template <typename T>
cudaError_t launch_gather(const GatherArgs &a, int d, int int4, cudaStream_t st)
{
    const dim3 grid((unsigned)((a.T + kGatherTokens - 1) / kGatherTokens), (unsigned)(2 * ((a.Hkv + kGatherRows - 1) / kGatherRows))), block(kGatherTokens * d / 8);
    LaunchScope scope(MOA_KERNEL_OTHER, st);
    if (d == 64)
        return int4 ? launch_dependent(kv_gather_kernel<T, 64, true>, grid, block, (size_t)0, st, a)
                    : launch_dependent(kv_gather_kernel<T, 64, false>, grid, block, (size_t)0, st, a);
    return int4 ? launch_dependent(kv_gather_kernel<T, 128, true>, grid, block, (size_t)0, st, a)
                : launch_dependent(kv_gather_kernel<T, 128, false>, grid, block, (size_t)0, st, a);
}

}  // namespace

cudaError_t kv_append(const AppendProblem &p, const void *q, const void *k, const void *v, const int *pos, const long long *slot,
                      const float *inv_freq, void *qo, void *pool, cudaStream_t st)
{
    AppendArgs a{};
    a.q = (const __nv_bfloat16 *)q; a.k = (const __nv_bfloat16 *)k; a.v = (const __nv_bfloat16 *)v;
    a.pos = pos; a.slot = slot; a.inv_freq = inv_freq; a.qo = (__nv_bfloat16 *)qo; a.pool = (uint8_t *)pool;
    a.sq = p.sq; a.sk = p.sk; a.sv = p.sv; a.so = p.so;
    a.page_stride = p.pool.page_stride;
    a.keys = (long long)p.pool.pages * p.pool.page;
    a.T = p.T; a.H = p.H; a.Hkv = p.pool.Hkv; a.page = p.pool.page; a.d_rot = p.d_rot;
    a.by_heads = FastDiv((uint32_t)(p.H > 0 ? p.H : 1));
    a.by_kv = FastDiv((uint32_t)p.pool.Hkv);
    a.by_page = FastDiv((uint32_t)p.pool.page);
    a.factor = p.factor;
    const int per = kThreads / (p.pool.d / 16), sms = device_info().sms;
    a.by_freqs = FastDiv((uint32_t)(p.d_rot > 0 ? p.d_rot / 2 : 1));
    a.tt = tokens_per_block(p.T, kTokens, kResident * sms);
    const int blocks = (p.T + a.tt - 1) / a.tt;
    // few tokens: keys and values in a block of their own, the queries in as many more as fill the SMs
    int split = 1;
    if (p.H > 0 && blocks < 2 * sms) {
        const int passes = (int)(((long long)a.tt * p.H + per - 1) / per);
        split = 2;
        while (split - 1 < passes && (long long)blocks * split < 2 * sms) ++split;
    }
    const dim3 grid((unsigned)blocks, (unsigned)split);
    if (p.pool.d == 64) return p.pool.int4 ? launch_append<64, true>(a, p.pairs, grid, st) : launch_append<64, false>(a, p.pairs, grid, st);
    return p.pool.int4 ? launch_append<128, true>(a, p.pairs, grid, st) : launch_append<128, false>(a, p.pairs, grid, st);
}

cudaError_t kv_gather(const CachePool &pool, int T, int dtype, const void *base, const long long *slot, void *k, void *v, RopeStride sk, RopeStride sv,
                      cudaStream_t st)
{
    GatherArgs a{};
    a.pool = (const uint8_t *)base; a.slot = slot; a.k = k; a.v = v; a.sk = sk; a.sv = sv;
    a.page_stride = pool.page_stride;
    a.keys = (long long)pool.pages * pool.page;
    a.T = T;
    a.Hkv = pool.Hkv; a.page = pool.page;
    a.by_page = FastDiv((uint32_t)pool.page);
    return dtype == MOA_F32 ? launch_gather<float>(a, pool.d, pool.int4, st) : launch_gather<__nv_bfloat16>(a, pool.d, pool.int4, st);
}

}  // namespace moa
