// What the rotary kernels (rope.cu) and the cache's append (cache.cu) share: angles, the rotation of the elements that a lane holds, and rows
// found without a division.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace moa {

// x / d for x < 2^31, by a product: (x * mul) >> 32 >> shift (Granlund and Montgomery's round-up method, 33-bit multiplier kept as 32 bits + 1)
struct FastDiv {
    uint32_t d, mul, shift;
    FastDiv() : FastDiv(1) {}
    explicit FastDiv(uint32_t div) : d(div), mul(0), shift(0)
    {
        while ((1ull << shift) < div) ++shift;
        mul = (uint32_t)((((1ull << shift) - div) << 32) / div + 1);
    }
    __host__ __device__ uint32_t div(uint32_t x) const
    {
#ifdef __CUDA_ARCH__
        const uint32_t hi = __umulhi(x, mul);
#else
        const uint32_t hi = (uint32_t)(((uint64_t)x * mul) >> 32);
#endif
        return (hi + x) >> shift;         // (hi <= x < 2^31: the sum has 32 bits)
    }
};

// pos * f, rounded to 64 bits (55 would be exact), as a part of a turn: 1 / (2 pi) in two parts, and what the product with the first one is rounded by, so
// that the farthest position loses nothing either (with one double for all of it, 2^31 radians were off by 5 * 2^-24)
__device__ __forceinline__ double part_of_turn(int pos, float f)
{
    const double a = (double)pos * (double)f, h = a * 0x1.45f306dc9c883p-3, l = fma(a, 0x1.45f306dc9c883p-3, -h) + a * -0x1.6b01ec5417056p-57;
    return (h - rint(h)) + l;
}

// cos and sin of pos * f, the product rounded to 64 bits.  What rounding the part of a turn to 32 bits takes off goes back in by the first term of the
// series: both results are within 1.5 * 2^-24.
__device__ __forceinline__ float2 position_angle(int pos, float f)
{
    const double t = part_of_turn(pos, f);
    const float h = (float)t, l = 6.2831853071795864769f * (float)(t - (double)h);
    float s, c;
    sincospif(2.f * h, &s, &c);
    return make_float2(fmaf(-l, s, c), fmaf(l, c, s));
}

// Sixteen bytes (or eight: V = 4 of bf16) of a row as floats, and back
template <typename T, int V> struct Chunk;
template <> struct Chunk<__nv_bfloat16, 8> {
    uint4 w;
    __device__ __forceinline__ void unpack(float (&f)[8]) const
    {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void pack(const float (&f)[8])
    {
        w = make_uint4(ptx::pack_bf16(f[0], f[1]), ptx::pack_bf16(f[2], f[3]), ptx::pack_bf16(f[4], f[5]), ptx::pack_bf16(f[6], f[7]));
    }
};
template <> struct Chunk<__nv_bfloat16, 4> {
    uint2 w;
    __device__ __forceinline__ void unpack(float (&f)[4]) const
    {
        f[0] = __uint_as_float(w.x << 16); f[1] = __uint_as_float(w.x & 0xffff0000u);
        f[2] = __uint_as_float(w.y << 16); f[3] = __uint_as_float(w.y & 0xffff0000u);
    }
    __device__ __forceinline__ void pack(const float (&f)[4]) { w = make_uint2(ptx::pack_bf16(f[0], f[1]), ptx::pack_bf16(f[2], f[3])); }
};
template <> struct Chunk<float, 4> {
    float4 w;
    __device__ __forceinline__ void unpack(float (&f)[4]) const { f[0] = w.x; f[1] = w.y; f[2] = w.z; f[3] = w.w; }
    __device__ __forceinline__ void pack(const float (&f)[4]) { w = make_float4(f[0], f[1], f[2], f[3]); }
};

// The lane's V pairs: (a[i], b[i]) in the half layout, neighbours of a and then of b in the other
template <int V, bool kPairs>
__device__ __forceinline__ void rotate(float (&a)[V], float (&b)[V], const float (&c)[V], const float (&s)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float &x = kPairs ? (i < V / 2 ? a[2 * i] : b[2 * i - V]) : a[i];
        float &y = kPairs ? (i < V / 2 ? a[2 * i + 1] : b[2 * i + 1 - V]) : b[i];
        const float x1 = x, x2 = y;
        x = fmaf(x1, c[i], -(x2 * s[i]));
        y = fmaf(x2, c[i], x1 * s[i]);
    }
}

// cos and sin of a token in shared memory: the V of a lane as V / 4 + V / 4 quads, quad-major over the `np` lanes of a row, so that neighbouring
// lanes read neighbouring quads
template <int V>
__device__ __forceinline__ void read_angles(const float4 *quads, int np, int p, float (&c)[V], float (&s)[V])
{
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const float4 x = quads[i * np + p], y = quads[(V / 4 + i) * np + p];
        c[4 * i] = x.x; c[4 * i + 1] = x.y; c[4 * i + 2] = x.z; c[4 * i + 3] = x.w;
        s[4 * i] = y.x; s[4 * i + 1] = y.y; s[4 * i + 2] = y.z; s[4 * i + 3] = y.w;
    }
}
template <int V>
__device__ __forceinline__ void write_angle(float4 *quads, int np, int freq, float2 cs)
{
    const int p = freq / V, i = freq % V;
    reinterpret_cast<float *>(quads + (i / 4) * np + p)[i % 4] = cs.x;
    reinterpret_cast<float *>(quads + (V / 4 + i / 4) * np + p)[i % 4] = cs.y;
}

// Tokens of a block, up to `most`: the fewest rounds of resident blocks, each as long as its tokens and the angles (about 0.7 of a token), so that
// the last round is not nearly empty.  (Equal shares for the resident blocks, gone through in such tiles, were 10 to 20 % slower: a block that waits
// for its next tile's angles has no other block behind it.)
inline int tokens_per_block(int T, int most, int resident)
{
    int best = 1;
    double cost = 0;
    for (int tt = 1; tt <= most; ++tt) {
        const int blocks = (T + tt - 1) / tt;
        const double c = (double)((blocks + resident - 1) / resident) * (tt + 0.7);
        if (tt == 1 || c < cost) { best = tt; cost = c; }
    }
    return best;
}

// rope.cu; strides {token, head} in elements (32 bits: an offset is two wide multiplications)
struct RopeStride {
    int token, head;
    __host__ __device__ __forceinline__ long long at(int t, int h) const { return (long long)t * token + (long long)h * head; }
};
struct RopeProblem {
    int T, H, Hk, d, d_rot, pairs;
    float factor;
    int backward;
    RopeStride sq, sk, so, sko;
};
cudaError_t rope(const RopeProblem &p, int dtype, const int *pos, const float *inv_freq, const void *q, const void *k, void *qo, void *ko,
                 cudaStream_t st);

}  // namespace moa
