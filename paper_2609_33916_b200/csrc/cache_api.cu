// C-ABI entry points of the rotary positions (include/moa_block.h) and the paged cache (include/moa_cache.h): argument checks.  No arithmetic here.
#include "cache_layout.cuh"
#include "moa_cache.h"

#include <cstddef>

using namespace moa;

// the layouts the Python binding mirrors
static_assert(sizeof(moa_rope_desc) == 96 && offsetof(moa_rope_desc, q_stride) == 32, "moa_rope_desc layout");
static_assert(sizeof(moa_cache_desc) == 32 && sizeof(moa_append_desc) == 120 && sizeof(moa_gather_desc) == 72 && sizeof(moa_paged_decode_desc) == 80,
              "cache descriptor layouts");

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned(const void *p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool finite(float v) { return v == v && v - v == 0.f; }

constexpr int kMostHeads = 1 << 16;
constexpr int64_t kMostStride = 1 << 30;

// {token, head} strides of T tokens x H heads x d; {0, 0} is [T,H,d].  Multiples of 16 bytes, at least d; an output's rows lie apart.
bool read_stride(const int64_t (&s)[2], int T, int H, int d, int elem, bool output, RopeStride *out)
{
    if (s[0] == 0 && s[1] == 0) {
        *out = RopeStride{H * d, d};
        return true;
    }
    if (s[0] < d || s[1] < d || s[0] % (16 / elem) != 0 || s[1] % (16 / elem) != 0) return false;
    if (s[0] > kMostStride || s[1] > kMostStride) return false;
    if (output && T > 1 && H > 1 && s[0] < (H - 1) * s[1] + d && s[1] < (T - 1) * s[0] + d) return false;
    *out = RopeStride{(int)s[0], (int)s[1]};
    return true;
}

moa_status check_rope(const moa_rope_desc *d, RopeProblem *p)
{
    if (!d) return MOA_ERR_INVALID_ARG;
    if (d->T <= 0 || d->H <= 0 || d->H_k < 0 || d->d <= 0 || d->d_rot <= 0 || d->d_rot > d->d) return MOA_ERR_INVALID_ARG;
    if (d->layout != MOA_ROPE_HALF && d->layout != MOA_ROPE_PAIRS) return MOA_ERR_INVALID_ARG;
    if (d->dtype != MOA_BF16 && d->dtype != MOA_F32) return MOA_ERR_INVALID_ARG;
    if (!finite(d->factor)) return MOA_ERR_INVALID_ARG;
    if (d->d % 8 != 0 || d->d > 256 || d->d_rot % 8 != 0 || d->H > kMostHeads || d->H_k > kMostHeads) return MOA_ERR_UNSUPPORTED;
    const int elem = d->dtype == MOA_F32 ? 4 : 2;
    *p = RopeProblem{};
    p->T = d->T; p->H = d->H; p->Hk = d->H_k; p->d = d->d; p->d_rot = d->d_rot;
    p->pairs = d->layout == MOA_ROPE_PAIRS;
    p->factor = d->factor;
    const int hk = d->H_k > 0 ? d->H_k : 1;
    if (!read_stride(d->q_stride, d->T, d->H, d->d, elem, false, &p->sq) || !read_stride(d->q_out_stride, d->T, d->H, d->d, elem, true, &p->so) ||
        !read_stride(d->k_stride, d->T, hk, d->d, elem, false, &p->sk) || !read_stride(d->k_out_stride, d->T, hk, d->d, elem, true, &p->sko))
        return MOA_ERR_INVALID_ARG;
    return MOA_OK;
}

moa_status rope_call(const moa_rope_desc *desc, int backward, const int32_t *pos, const float *inv_freq, const void *q, const void *k, void *qo,
                     void *ko, void *stream)
{
    RopeProblem p;
    moa_status s = check_rope(desc, &p);
    if (s != MOA_OK) return s;
    if (!pos || !inv_freq || !q || !qo || (p.Hk > 0 && (!k || !ko))) return MOA_ERR_INVALID_ARG;
    if (!aligned(pos, 4) || !aligned(inv_freq, 4) || !aligned16(q) || !aligned16(qo)) return MOA_ERR_INVALID_ARG;
    if (p.Hk > 0 && (!aligned16(k) || !aligned16(ko))) return MOA_ERR_INVALID_ARG;
    // in place means the same rows
    if (q == qo && (p.sq.token != p.so.token || p.sq.head != p.so.head)) return MOA_ERR_INVALID_ARG;
    if (p.Hk > 0 && k == ko && (p.sk.token != p.sko.token || p.sk.head != p.sko.head)) return MOA_ERR_INVALID_ARG;
    if ((s = check_device_arch()) != MOA_OK) return s;
    p.backward = backward;
    return rope(p, desc->dtype, pos, inv_freq, q, k, qo, ko, (cudaStream_t)stream) == cudaSuccess ? MOA_OK : MOA_ERR_CUDA;
}

moa_status check_cache(const moa_cache_desc *d, CachePool *p)
{
    if (d->pages <= 0 || d->page <= 0 || d->H_kv <= 0 || d->d <= 0 || d->reserved != 0 || d->page_stride < 0) return MOA_ERR_INVALID_ARG;
    if (d->format != MOA_CACHE_BF16 && d->format != MOA_CACHE_INT4) return MOA_ERR_INVALID_ARG;
    if (d->page % kBlockKeys != 0 || d->page > 1024 || (d->d != 64 && d->d != 128) || d->H_kv > kMostHeads) return MOA_ERR_UNSUPPORTED;
    *p = CachePool{d->pages, d->page, d->H_kv, d->d, d->format == MOA_CACHE_INT4, d->page_stride};
    if (d->page_stride != 0 && (d->page_stride % 16 != 0 || d->page_stride < p->page_bytes() || d->page_stride > (1LL << 40))) return MOA_ERR_INVALID_ARG;
    if (d->page_stride == 0) p->page_stride = p->page_bytes();
    return MOA_OK;
}

moa_status check_append(const moa_append_desc *d, AppendProblem *p)
{
    if (!d) return MOA_ERR_INVALID_ARG;
    *p = AppendProblem{};
    const moa_status s = check_cache(&d->cache, &p->pool);
    if (s != MOA_OK) return s;
    if (d->T <= 0 || d->H < 0 || d->d_rot < 0 || d->d_rot > d->cache.d) return MOA_ERR_INVALID_ARG;
    if (d->layout != MOA_ROPE_HALF && d->layout != MOA_ROPE_PAIRS) return MOA_ERR_INVALID_ARG;
    if (d->dtype != MOA_BF16 && d->dtype != MOA_F32) return MOA_ERR_INVALID_ARG;
    if (!finite(d->factor) || (d->d_rot == 0 && d->H > 0)) return MOA_ERR_INVALID_ARG;
    if (d->dtype != MOA_BF16 || d->d_rot % 16 != 0 || d->H > kMostHeads) return MOA_ERR_UNSUPPORTED;
    p->T = d->T; p->H = d->H; p->d_rot = d->d_rot;
    p->pairs = d->layout == MOA_ROPE_PAIRS;
    p->factor = d->factor;
    const int hd = d->cache.d, hk = d->cache.H_kv, hq = d->H > 0 ? d->H : 1;
    if (!read_stride(d->q_stride, d->T, hq, hd, 2, false, &p->sq) || !read_stride(d->q_out_stride, d->T, hq, hd, 2, true, &p->so) ||
        !read_stride(d->k_stride, d->T, hk, hd, 2, false, &p->sk) || !read_stride(d->v_stride, d->T, hk, hd, 2, false, &p->sv))
        return MOA_ERR_INVALID_ARG;
    return MOA_OK;
}

moa_status check_paged(const moa_paged_decode_desc *d, PagedProblem *p)
{
    if (!d) return MOA_ERR_INVALID_ARG;
    *p = PagedProblem{};
    const moa_status s = check_cache(&d->cache, &p->pool);
    if (s != MOA_OK) return s;
    if (d->B <= 0 || d->H <= 0 || d->max_pages <= 0 || d->reserved != 0 || d->table_stride < 0) return MOA_ERR_INVALID_ARG;
    if (d->H % d->cache.H_kv != 0 || (d->table_stride != 0 && d->table_stride < d->max_pages)) return MOA_ERR_INVALID_ARG;
    if (d->dtype != MOA_BF16 && d->dtype != MOA_F32) return MOA_ERR_INVALID_ARG;
    if (!finite(d->scale)) return MOA_ERR_INVALID_ARG;
    if (d->dtype != MOA_BF16 || d->H / d->cache.H_kv > 16 || d->scale > 0x1p60f || d->scale < -0x1p60f) return MOA_ERR_UNSUPPORTED;
    // keys of a row of the table, and units of 64 keys of all rows, are counted in 32 bits
    const long long cap = (long long)d->max_pages * d->cache.page;
    if (cap > (1LL << 30) || (cap + 63) / 64 * d->cache.H_kv > (1LL << 30) / d->B || d->table_stride > (1LL << 40)) return MOA_ERR_UNSUPPORTED;
    p->B = d->B; p->H = d->H; p->max_pages = d->max_pages;
    p->scale = d->scale;
    p->table_stride = d->table_stride ? d->table_stride : d->max_pages;
    if (!read_stride(d->q_stride, d->B, d->H, d->cache.d, 2, false, &p->sq)) return MOA_ERR_INVALID_ARG;
    return MOA_OK;
}

}  // namespace

extern "C" {

moa_status moa_rope_fwd(const moa_rope_desc *desc, const int32_t *pos, const float *inv_freq, const void *q, const void *k, void *q_out, void *k_out,
                        void *stream)
{
    return rope_call(desc, 0, pos, inv_freq, q, k, q_out, k_out, stream);
}

moa_status moa_rope_bwd(const moa_rope_desc *desc, const int32_t *pos, const float *inv_freq, const void *dq, const void *dk, void *dq_in, void *dk_in,
                        void *stream)
{
    return rope_call(desc, 1, pos, inv_freq, dq, dk, dq_in, dk_in, stream);
}

size_t moa_cache_page_bytes(const moa_cache_desc *desc)
{
    CachePool p;
    return desc && check_cache(desc, &p) == MOA_OK ? (size_t)p.page_bytes() : 0;
}

moa_status moa_kv_append(const moa_append_desc *desc, const void *q, const void *k, const void *v, const int32_t *pos, const int64_t *slot,
                         const float *inv_freq, void *q_out, void *pool, void *stream)
{
    AppendProblem p;
    moa_status s = check_append(desc, &p);
    if (s != MOA_OK) return s;
    if (!k || !v || !slot || !pool || (p.H > 0 && (!q || !q_out)) || (p.d_rot > 0 && (!pos || !inv_freq))) return MOA_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || !aligned16(pool) || !aligned(slot, 8) || !aligned(pos, 4) || !aligned(inv_freq, 4)) return MOA_ERR_INVALID_ARG;
    if (p.H > 0 && (!aligned16(q) || !aligned16(q_out))) return MOA_ERR_INVALID_ARG;
    if (p.H > 0 && q == q_out && (p.sq.token != p.so.token || p.sq.head != p.so.head)) return MOA_ERR_INVALID_ARG;
    if ((s = check_device_arch()) != MOA_OK) return s;
    return kv_append(p, q, k, v, pos, (const long long *)slot, inv_freq, q_out, pool, (cudaStream_t)stream) == cudaSuccess ? MOA_OK : MOA_ERR_CUDA;
}

moa_status moa_kv_gather(const moa_gather_desc *desc, const void *pool, const int64_t *slot, void *k, void *v, void *stream)
{
    if (!desc) return MOA_ERR_INVALID_ARG;
    CachePool p{};
    moa_status s = check_cache(&desc->cache, &p);
    if (s != MOA_OK) return s;
    if (desc->T <= 0 || (desc->dtype != MOA_BF16 && desc->dtype != MOA_F32)) return MOA_ERR_INVALID_ARG;
    RopeStride sk, sv;
    const int elem = desc->dtype == MOA_F32 ? 4 : 2;
    if (!read_stride(desc->k_stride, desc->T, p.Hkv, p.d, elem, true, &sk) || !read_stride(desc->v_stride, desc->T, p.Hkv, p.d, elem, true, &sv))
        return MOA_ERR_INVALID_ARG;
    if (!pool || !slot || !k || !v) return MOA_ERR_INVALID_ARG;
    if (!aligned16(pool) || !aligned(slot, 8) || !aligned16(k) || !aligned16(v)) return MOA_ERR_INVALID_ARG;
    if ((s = check_device_arch()) != MOA_OK) return s;
    return kv_gather(p, desc->T, desc->dtype, pool, (const long long *)slot, k, v, sk, sv, (cudaStream_t)stream) == cudaSuccess ? MOA_OK : MOA_ERR_CUDA;
}

size_t moa_paged_decode_workspace_bytes(const moa_paged_decode_desc *desc)
{
    PagedProblem p;
    return check_paged(desc, &p) == MOA_OK ? paged_decode_workspace_bytes(p) : 0;
}

moa_status moa_paged_decode(const moa_paged_decode_desc *desc, const void *q, const void *pool, const int32_t *table, const int32_t *lens, void *out,
                            float *lse, void *ws, size_t ws_bytes, void *stream)
{
    PagedProblem p;
    moa_status s = check_paged(desc, &p);
    if (s != MOA_OK) return s;
    if (!q || !pool || !table || !lens || !out) return MOA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(pool) || !aligned(table, 4) || !aligned(lens, 4) || !aligned16(out) || !aligned(lse, 4)) return MOA_ERR_INVALID_ARG;
    if (!ws || ws_bytes < paged_decode_workspace_bytes(p)) return MOA_ERR_WORKSPACE;
    if (!aligned16(ws)) return MOA_ERR_INVALID_ARG;
    if ((s = check_device_arch()) != MOA_OK) return s;
    return paged_decode(p, q, pool, table, lens, out, lse, ws, (cudaStream_t)stream) == cudaSuccess ? MOA_OK : MOA_ERR_CUDA;
}

}  // extern "C"
