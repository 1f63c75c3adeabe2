// Rotary positions of queries and keys, forward and backward (the transposed rotation: the sine's sign).
//
// HBM-bound: every element is read and written once, 6 flop per pair.  The angles are the only other work: d_rot / 2 of them per token, each
// a 64-bit product and a sine and cosine of about 60 instructions, against H + H_k heads that share them.  So a block takes up to four
// tokens with all their heads, makes each angle once (one per thread at d_rot = 128) and keeps them in shared memory; a row of a head is then
// d / 16 lanes with the two 16-byte pieces of it that rotate into each other, two rows in flight per lane.
// No table of angles: one would be read per token and head size, needs a largest position, and is not faster than what hides under the
// loads here.
#include "rotate.cuh"

namespace moa {
namespace {

using namespace ptx;

constexpr int kThreads = 256, kTokens = 4, kUnroll = 2, kResident = 5;

struct RopeArgs {
    const int *pos;
    const float *inv_freq;
    const void *q, *k;
    void *qo, *ko;
    RopeStride sq, sk, so, sko;
    int T, H, d, d_rot, tt;      // tt: tokens per block
    int lanes, np;               // lanes per row; those of them that rotate
    FastDiv rows, by_lanes, by_freqs;      // heads of q and k, lanes, d_rot / 2
    float factor, sign;
};

template <typename T, int V, bool kPairs>
__global__ void __launch_bounds__(kThreads, kResident) rope_kernel(const RopeArgs a)
{
    __shared__ float4 angles[kTokens * 64];      // (256 elements: 128 angles of 8 bytes per token)
    const int tid = threadIdx.x, t0 = blockIdx.x * a.tt, nt = min(a.tt, a.T - t0), freqs = a.d_rot / 2;
    grid_dependency_wait();
    grid_launch_dependents();
    const int *pos = after_wait(a.pos);
    const float *inv_freq = after_wait(a.inv_freq);
    for (int i = tid; i < nt * freqs; i += kThreads) {
        const int t = (int)a.by_freqs.div((uint32_t)i), f = i - t * freqs;
        float2 cs = position_angle(pos[t0 + t], inv_freq[f]);
        cs.x *= a.factor;
        cs.y *= a.factor * a.sign;
        write_angle<V>(angles + t * (freqs / 2), a.np, f, cs);
    }
    __syncthreads();
    const int r0 = (int)a.by_lanes.div((uint32_t)tid), p = tid - r0 * a.lanes, per = kThreads / a.lanes;
    if (r0 >= per) return;
    const bool turns = p < a.np;
    const int c0 = turns && !kPairs ? p * V : 2 * p * V, c1 = turns && !kPairs ? freqs + p * V : c0 + V;
    const bool two = c1 < a.d;       // (what is not turned may end with a single piece)
    const int total = nt * (int)a.rows.d;
    const T *q = after_wait((const T *)a.q), *k = after_wait((const T *)a.k);
    for (int r = r0 + (int)blockIdx.y * per * kUnroll; r < total; r += per * kUnroll * (int)gridDim.y) {
        Chunk<T, V> x[kUnroll], y[kUnroll];
        T *dst[kUnroll];
        int tok[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int row = r + u * per;
            dst[u] = nullptr;
            if (row < total) {
                tok[u] = (int)a.rows.div((uint32_t)row);
                const int h = row - tok[u] * (int)a.rows.d;
                const int t = t0 + tok[u];
                const T *src;
                if (h < a.H) {
                    src = q + a.sq.at(t, h);
                    dst[u] = (T *)a.qo + a.so.at(t, h);
                } else {
                    src = k + a.sk.at(t, h - a.H);
                    dst[u] = (T *)a.ko + a.sko.at(t, h - a.H);
                }
                x[u] = *reinterpret_cast<const Chunk<T, V> *>(src + c0);
                if (two) y[u] = *reinterpret_cast<const Chunk<T, V> *>(src + c1);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (!dst[u]) continue;
            if (turns) {
                float fx[V], fy[V], c[V], s[V];
                read_angles<V>(angles + tok[u] * (freqs / 2), a.np, p, c, s);
                x[u].unpack(fx);
                y[u].unpack(fy);
                rotate<V, kPairs>(fx, fy, c, s);
                x[u].pack(fx);
                y[u].pack(fy);
            }
            *reinterpret_cast<Chunk<T, V> *>(dst[u] + c0) = x[u];
            if (two) *reinterpret_cast<Chunk<T, V> *>(dst[u] + c1) = y[u];
        }
    }
}

template <typename T, int V>
cudaError_t launch(const RopeProblem &p, const int *pos, const float *inv_freq, const void *q, const void *k, void *qo, void *ko, cudaStream_t st)
{
    RopeArgs a{};
    a.pos = pos; a.inv_freq = inv_freq; a.q = q; a.k = k; a.qo = qo; a.ko = ko;
    a.sq = p.sq; a.sk = p.sk; a.so = p.so; a.sko = p.sko;
    a.T = p.T; a.H = p.H; a.d = p.d; a.d_rot = p.d_rot;
    a.np = p.d_rot / (2 * V);
    // in place, what is not turned stays where it is
    const bool in_place = q == qo && (p.Hk == 0 || k == ko);
    a.lanes = in_place ? a.np : a.np + (p.d - p.d_rot + 2 * V - 1) / (2 * V);
    const int rows = p.H + p.Hk, per = kThreads / a.lanes, sms = device_info().sms;
    a.rows = FastDiv((uint32_t)rows);
    a.by_lanes = FastDiv((uint32_t)a.lanes);
    a.factor = p.factor;
    a.sign = p.backward ? -1.f : 1.f;
    // a few tokens: one to a block, and its rows over several
    a.by_freqs = FastDiv((uint32_t)(p.d_rot / 2));
    a.tt = tokens_per_block(p.T, kTokens, kResident * sms);
    const int blocks = (p.T + a.tt - 1) / a.tt, passes = (a.tt * rows + per * kUnroll - 1) / (per * kUnroll);
    int split = 1;
    while (split < passes && blocks * split < 2 * sms) ++split;
    LaunchScope scope(MOA_KERNEL_OTHER, st);
    const dim3 grid((unsigned)blocks, (unsigned)split);
    return p.pairs ? launch_dependent(rope_kernel<T, V, true>, grid, dim3(kThreads), (size_t)0, st, a)
                   : launch_dependent(rope_kernel<T, V, false>, grid, dim3(kThreads), (size_t)0, st, a);
}

}  // namespace

cudaError_t rope(const RopeProblem &p, int dtype, const int *pos, const float *inv_freq, const void *q, const void *k, void *qo, void *ko,
                 cudaStream_t st)
{
    if (dtype == MOA_F32) return launch<float, 4>(p, pos, inv_freq, q, k, qo, ko, st);
    // pieces of 16 bytes where the halves are made of them (d_rot a multiple of 16)
    return p.d_rot % 16 == 0 ? launch<__nv_bfloat16, 8>(p, pos, inv_freq, q, k, qo, ko, st)
                             : launch<__nv_bfloat16, 4>(p, pos, inv_freq, q, k, qo, ko, st);
}

}  // namespace moa
