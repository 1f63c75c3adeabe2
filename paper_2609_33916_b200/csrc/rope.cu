// Rotary positions of queries and keys, forward and backward (the transposed rotation: the sine's sign).
//
// HBM-bound: every element is read and written once, 6 flop per pair.  The angles are the only other work: d_rot / 2 of them per token, each
// a 64-bit product and a sine and cosine of about 60 instructions, against H + H_k heads that share them.  So a block of two warps takes a token
// with all its heads, makes each angle once (one per thread at d_rot = 128) and keeps them in shared memory; a row of a head is then d / 16 lanes with
// the two 16-byte pieces of it that rotate into each other, two rows in flight per lane.  Small blocks, twenty to an SM: while one makes its angles others
// stream, and the last round of blocks is short; the first rows are on their way while the angles are made (B2 n4096 H16/16 d128, 134 MB: 22.6 us, 5.9 TB/s;
// with the loads behind the angles 23.5, with 16 or 18 blocks to an SM 23.2 and 23.9, four tokens to 256 threads 23.8; 3001 tokens of
// fp32 H8/2 d80 4.1, behind the angles 4.6; equal shares of the tokens for the resident blocks 25; four rows in flight 24.0).
// No table of angles: one would be read per token and head size, needs a largest position, and is not faster than what hides under the
// loads here.
#include "rotate.cuh"

namespace moa {
namespace {

using namespace ptx;

constexpr int kThreads = 64, kUnroll = 2, kResident = 20;

struct RopeArgs {
    const int *pos;
    const float *inv_freq;
    const void *q, *k;
    void *qo, *ko;
    RopeStride sq, sk, so, sko;
    int H, rows, d, d_rot;       // rows: heads of q and k
    int lanes, np;               // lanes per row; those of them that rotate
    FastDiv by_lanes;
    float factor, sign;
};

// blockIdx.x: the token; its rows are shared by gridDim.y blocks
template <typename T, int V, bool kPairs>
__global__ void __launch_bounds__(kThreads, kResident) rope_kernel(const RopeArgs a)
{
    __shared__ float4 angles[64];      // (256 elements: 128 angles of 8 bytes)
    const int tid = threadIdx.x, t = blockIdx.x, freqs = a.d_rot / 2;
    grid_dependency_wait();
    grid_launch_dependents();
    const int at = after_wait(a.pos)[t];
    const float *inv_freq = after_wait(a.inv_freq);
    const int r0 = (int)a.by_lanes.div((uint32_t)tid), p = tid - r0 * a.lanes, per = kThreads / a.lanes;
    const bool turns = p < a.np;
    const int c0 = turns && !kPairs ? p * V : 2 * p * V, c1 = turns && !kPairs ? freqs + p * V : c0 + V;
    const bool two = c1 < a.d;       // (what is not turned may end with a single piece)
    const int rows = r0 < per ? a.rows : 0;
    const T *q = after_wait((const T *)a.q) + (long long)t * a.sq.token, *k = after_wait((const T *)a.k) + (long long)t * a.sk.token;
    T *qo = (T *)a.qo + (long long)t * a.so.token, *ko = (T *)a.ko + (long long)t * a.sko.token;
    Chunk<T, V> x[kUnroll], y[kUnroll];
    auto load = [&](int r) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = r + u * per, hk = h - a.H;
            if (h < rows) {
                const T *src = hk < 0 ? q + (long long)h * a.sq.head : k + (long long)hk * a.sk.head;
                x[u] = *reinterpret_cast<const Chunk<T, V> *>(src + c0);
                if (two) y[u] = *reinterpret_cast<const Chunk<T, V> *>(src + c1);
            }
        }
    };
    int r = r0 + (int)blockIdx.y * per * kUnroll;
    load(r);
    for (int f = tid; f < freqs; f += kThreads) {
        float2 cs = position_angle(at, inv_freq[f]);
        cs.x *= a.factor;
        cs.y *= a.factor * a.sign;
        write_angle<V>(angles, a.np, f, cs);
    }
    __syncthreads();
    while (r < rows) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = r + u * per, hk = h - a.H;
            if (h >= rows) continue;
            T *dst = hk < 0 ? qo + (long long)h * a.so.head : ko + (long long)hk * a.sko.head;
            if (turns) {
                float fx[V], fy[V], c[V], s[V];
                read_angles<V>(angles, a.np, p, c, s);
                x[u].unpack(fx);
                y[u].unpack(fy);
                rotate<V, kPairs>(fx, fy, c, s);
                x[u].pack(fx);
                y[u].pack(fy);
            }
            *reinterpret_cast<Chunk<T, V> *>(dst + c0) = x[u];
            if (two) *reinterpret_cast<Chunk<T, V> *>(dst + c1) = y[u];
        }
        r += per * kUnroll * (int)gridDim.y;
        load(r);
    }
}

template <typename T, int V>
cudaError_t launch(const RopeProblem &p, const int *pos, const float *inv_freq, const void *q, const void *k, void *qo, void *ko, cudaStream_t st)
{
    RopeArgs a{};
    a.pos = pos; a.inv_freq = inv_freq; a.q = q; a.k = k; a.qo = qo; a.ko = ko;
    a.sq = p.sq; a.sk = p.sk; a.so = p.so; a.sko = p.sko;
    a.H = p.H; a.rows = p.H + p.Hk; a.d = p.d; a.d_rot = p.d_rot;
    a.np = p.d_rot / (2 * V);
    // in place, what is not turned stays where it is
    const bool in_place = q == qo && (p.Hk == 0 || k == ko);
    a.lanes = in_place ? a.np : a.np + (p.d - p.d_rot + 2 * V - 1) / (2 * V);
    a.by_lanes = FastDiv((uint32_t)a.lanes);
    a.factor = p.factor;
    a.sign = p.backward ? -1.f : 1.f;
    // fewer tokens than three quarters of what is resident: their rows over several blocks each (1598 tokens H16/4 d256: 7.2 us, in one block each 10.2)
    const int per = kThreads / a.lanes, passes = (a.rows + per * kUnroll - 1) / (per * kUnroll), sms = device_info().sms;
    int split = 1;
    while (split < passes && (long long)p.T * split * 4 < 3LL * kResident * sms) ++split;
    LaunchScope scope(MOA_KERNEL_OTHER, st);
    const dim3 grid((unsigned)p.T, (unsigned)split);
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
