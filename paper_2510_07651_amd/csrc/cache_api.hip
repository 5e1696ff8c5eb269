// Host side of the cache calls of the C ABI (obc_cache_append, obc_attend, obc_cache_read): argument checks and dispatch.
// Nothing here allocates or synchronises.
#include <cmath>
#include <cstring>
#include <utility>

#include "cache.h"

namespace obc {
namespace {

size_t element_bytes(int dtype) { return dtype == OBC_F32 ? 4 : dtype == OBC_BF16 ? 2 : 1; }

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int check_cache(const obc_cache_t *c, CacheView *view) {
    if (!c) return OBC_EINVAL;
    if (!c->k || !c->v || c->num_pages < 1 || c->pages_per_seq < 1 || c->page_size < 1 || c->batch < 1 || c->Hkv < 1 || c->d < 1)
        return OBC_EINVAL;
    if (c->dtype != OBC_F32 && c->dtype != OBC_BF16 && c->dtype != OBC_E4M3) return OBC_EUNSUPPORTED;
    if (c->d != 64 && c->d != 128) return OBC_EUNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->page_table, 4)) return OBC_EINVAL;
    if (c->dtype == OBC_E4M3) {
        if (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16)) return OBC_EINVAL;
    } else if (c->k_scale || c->v_scale) {
        return OBC_EINVAL;
    }
    int shift = 31;
    if (c->page_table) {
        if ((c->page_size & (c->page_size - 1)) != 0) return OBC_EUNSUPPORTED;
        shift = __builtin_ctz((unsigned)c->page_size);
    } else if (c->batch != c->num_pages || c->pages_per_seq != 1) {
        return OBC_EINVAL;
    }
    const long long capacity = (long long)c->pages_per_seq * c->page_size;
    if (capacity > OBC_MAX_CACHE_ROWS || (long long)c->batch * c->Hkv > 65535) return OBC_EUNSUPPORTED;
    *view = {(char *)c->k, (char *)c->v, c->k_scale, c->v_scale, c->page_table, c->num_pages, c->pages_per_seq, c->page_size, shift,
             c->Hkv, (int)capacity};
    return OBC_OK;
}

// Rows of d elements that may be read 16 bytes at a time.  The stride of a dimension of size 1 is nobody's: 0 in the view.
int check_rows(const obc_rows_t *r, int B, int T, int H, int dtype, RowsView *view) {
    if (!r || !r->data || !aligned(r->data, 16)) return OBC_EINVAL;
    const int64_t size = (int64_t)element_bytes(dtype), most = INT64_MAX / 64;
    const int64_t strides[3] = {B > 1 ? r->batch_stride : 0, T > 1 ? r->token_stride : 0, H > 1 ? r->head_stride : 0};
    for (const int64_t s : strides)
        if (s < 0 || s > most || s * size % 16 != 0) return OBC_EINVAL;
    *view = {(const char *)r->data, strides[0] * size, strides[1] * size, strides[2] * size};
    return OBC_OK;
}

bool overlap(const void *p, const void *q, int64_t p_bytes, int64_t q_bytes) {
    return (uintptr_t)p < (uintptr_t)q + (uintptr_t)q_bytes && (uintptr_t)q < (uintptr_t)p + (uintptr_t)p_bytes;
}

// Whether one of the rows (of `row` bytes) meets the `bytes` from `p` on.  Rows that are apart from them as a whole, which is all but every
// call, cost three products; others are gone through, two dimensions step by step, the longest at once.
bool meets_rows(const RowsView &r, int B, int T, int H, int64_t row, const void *p, int64_t bytes) {
    typedef __int128 wide;
    struct { int64_t n, stride; } dim[3] = {{B, r.batch}, {T, r.token}, {H, r.head}};
    const wide from = (wide)(uintptr_t)p - (wide)(uintptr_t)r.base, to = from + bytes;
    if (to <= 0 || from >= (wide)(B - 1) * r.batch + (wide)(T - 1) * r.token + (wide)(H - 1) * r.head + row) return false;
    if (dim[0].n > dim[2].n) std::swap(dim[0], dim[2]);
    if (dim[1].n > dim[2].n) std::swap(dim[1], dim[2]);
    for (int64_t i = 0; i < dim[0].n; ++i)
        for (int64_t j = 0; j < dim[1].n; ++j) {
            // the first row that ends behind `from`
            const wide at = (wide)i * dim[0].stride + (wide)j * dim[1].stride, short_by = from - row + 1 - at;
            const wide k = short_by <= 0 ? 0 : dim[2].stride == 0 ? dim[2].n : (short_by + dim[2].stride - 1) / dim[2].stride;
            if (k < dim[2].n && at + k * dim[2].stride < to) return true;
        }
    return false;
}

int attend_plan_of(int B, int T, int Hq, const obc_cache_t *cache, int dtype, CacheView *view, AttendPlan *plan) {
    const int rc = check_cache(cache, view);
    if (rc != OBC_OK) return rc;
    if (B != cache->batch || T < 1 || Hq < 1 || Hq % cache->Hkv != 0) return OBC_EINVAL;
    if (dtype != OBC_F32 && dtype != OBC_BF16) return OBC_EUNSUPPORTED;
    if (cache->dtype != dtype && cache->dtype != OBC_E4M3) return OBC_EUNSUPPORTED;
    if ((long long)Hq / cache->Hkv * T > (1LL << 24) || (long long)B * Hq * T > (1LL << 28)) return OBC_EUNSUPPORTED;
    plan_attend(B, T, Hq, cache->Hkv, cache->d, view->capacity, dtype, cache->dtype, plan);
    return OBC_OK;
}

}  // namespace
}  // namespace obc

using namespace obc;

extern "C" {

int obc_cache_append(const obc_rows_t *q, const obc_rows_t *k, const obc_rows_t *v, const obc_cache_t *cache, void *q_out,
                     const int32_t *lens, int lens_per_head, const int32_t *new_lens, int new_lens_per_head,
                     const int32_t *positions, const float *inv_freq, int rot_pairs, float rot_scale, int interleaved,
                     const void *q_norm, const void *k_norm, float eps, int B, int T, int Hq, int dtype, void *hip_stream) {
    AppendArgs a;
    std::memset(&a, 0, sizeof(a));
    int rc = check_cache(cache, &a.cache);
    if (rc != OBC_OK) return rc;
    if (B != cache->batch || T < 1 || !lens) return OBC_EINVAL;
    if (dtype != OBC_F32 && dtype != OBC_BF16) return OBC_EUNSUPPORTED;
    if (cache->dtype != dtype && cache->dtype != OBC_E4M3) return OBC_EUNSUPPORTED;
    if ((rc = check_rows(k, B, T, cache->Hkv, dtype, &a.k)) != OBC_OK || (rc = check_rows(v, B, T, cache->Hkv, dtype, &a.v)) != OBC_OK) return rc;
    if (q) {
        if ((rc = check_rows(q, B, T, Hq, dtype, &a.q)) != OBC_OK) return rc;
        if (!q_out || !aligned(q_out, 16) || Hq < 1 || Hq % cache->Hkv != 0) return OBC_EINVAL;
        if (new_lens && new_lens_per_head) return OBC_EINVAL;      // a query belongs to its token, not to a KV head's list
    } else if (q_out || q_norm || Hq != 0) {
        return OBC_EINVAL;
    }
    if (rot_pairs < 0 || 2 * (long long)rot_pairs > cache->d) return OBC_EINVAL;
    if (rot_pairs % 8 != 0) return OBC_EUNSUPPORTED;
    if (rot_pairs > 0 && (!positions || !inv_freq || !std::isfinite(rot_scale))) return OBC_EINVAL;
    if (!aligned(lens, 4) || !aligned(new_lens, 4) || !aligned(positions, 4) || !aligned(inv_freq, 4) || !aligned(q_norm, 16) ||
        !aligned(k_norm, 16))
        return OBC_EINVAL;
    if ((q_norm || k_norm) && !(eps >= 0.f && std::isfinite(eps))) return OBC_EINVAL;
    // A grid holds fewer than 2^32 threads: with norm, rotation or queries a workgroup of 256 per token, else one per 16 rows.
    const bool as_they_are = !q && !rot_pairs && !k_norm;
    if ((long long)B * T >= (as_they_are ? 1LL << 27 : 1LL << 24) || (long long)B * T * (Hq + 2LL * cache->Hkv) > (1LL << 34) || Hq > 65535)
        return OBC_EUNSUPPORTED;
    if (q) {
        const int64_t row = cache->d * (int64_t)element_bytes(dtype), out = (int64_t)B * T * Hq * row;
        if (meets_rows(a.q, B, T, Hq, row, q_out, out) || meets_rows(a.k, B, T, cache->Hkv, row, q_out, out) ||
            meets_rows(a.v, B, T, cache->Hkv, row, q_out, out))
            return OBC_EINVAL;
    }
    a.q_out = (char *)q_out;
    a.lens = {lens, lens_per_head != 0};
    a.fresh = {new_lens, new_lens_per_head != 0};
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.pairs = rot_pairs;
    a.rot_scale = rot_scale;
    a.interleaved = interleaved != 0;
    a.q_norm = q_norm;
    a.k_norm = k_norm;
    a.eps = eps;
    a.B = B; a.T = T; a.Hq = Hq; a.d = cache->d; a.dtype = dtype; a.cache_dtype = cache->dtype;
    return launch_append(a, (hipStream_t)hip_stream) == hipSuccess ? OBC_OK : OBC_ELAUNCH;
}

int obc_attend_workspace_bytes(int B, int T, int Hq, const obc_cache_t *cache, int dtype, size_t *bytes_out) {
    if (!bytes_out) return OBC_EINVAL;
    CacheView view;
    AttendPlan plan;
    const int rc = attend_plan_of(B, T, Hq, cache, dtype, &view, &plan);
    if (rc != OBC_OK) return rc;
    *bytes_out = plan.total;
    return OBC_OK;
}

int obc_attend(const void *q, const obc_cache_t *cache, void *out, const int32_t *lens, int lens_per_head, const int32_t *new_lens,
               int B, int T, int Hq, int dtype, int causal, float scale, void *workspace, size_t workspace_bytes, void *hip_stream) {
    AttendArgs a;
    AttendPlan plan;
    std::memset(&a, 0, sizeof(a));
    const int rc = attend_plan_of(B, T, Hq, cache, dtype, &a.cache, &plan);
    if (rc != OBC_OK) return rc;
    if (!q || !out || !lens || !aligned(q, 16) || !aligned(out, 16) || !aligned(lens, 4) || !aligned(new_lens, 4)) return OBC_EINVAL;
    if (!(scale > 0.f) || !std::isfinite(scale * 1.4426950408889634f)) return OBC_EINVAL;
    if (plan.total && (!workspace || !aligned(workspace, 256) || workspace_bytes < plan.total)) return OBC_EWORKSPACE;
    const int64_t rows_bytes = (int64_t)B * T * Hq * cache->d * (int64_t)element_bytes(dtype);
    if (overlap(q, out, rows_bytes, rows_bytes)) return OBC_EINVAL;
    a.q = (const char *)q;
    a.out = (char *)out;
    a.lens = {lens, lens_per_head != 0};
    a.fresh = new_lens;
    a.B = B; a.T = T; a.Hq = Hq; a.Hkv = cache->Hkv; a.G = Hq / cache->Hkv; a.d = cache->d;
    a.dtype = dtype; a.cache_dtype = cache->dtype;
    a.causal = causal != 0;
    a.scale_log2 = scale * 1.4426950408889634f;
    return launch_attend(a, plan, (char *)workspace, (hipStream_t)hip_stream) == hipSuccess ? OBC_OK : OBC_ELAUNCH;
}

int obc_cache_read(const obc_cache_t *cache, const int32_t *keep_idx, void *k_out, void *v_out, int B, int n, int dtype, void *hip_stream) {
    ReadArgs a;
    std::memset(&a, 0, sizeof(a));
    const int rc = check_cache(cache, &a.cache);
    if (rc != OBC_OK) return rc;
    if (B != cache->batch || n < 1 || (!keep_idx && n > a.cache.capacity)) return OBC_EINVAL;
    if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(keep_idx, 4)) return OBC_EINVAL;
    if (dtype != OBC_F32 && dtype != OBC_BF16) return OBC_EUNSUPPORTED;
    if (cache->dtype != dtype && cache->dtype != OBC_E4M3) return OBC_EUNSUPPORTED;
    if (n > OBC_MAX_CACHE_ROWS / 8 || (long long)B * cache->Hkv * n > (1LL << 34)) return OBC_EUNSUPPORTED;
    const int64_t out_bytes = (int64_t)B * cache->Hkv * n * cache->d * (int64_t)element_bytes(dtype);
    if (overlap(k_out, v_out, out_bytes, out_bytes)) return OBC_EINVAL;
    a.keep = keep_idx;
    a.k_out = (char *)k_out;
    a.v_out = (char *)v_out;
    a.B = B; a.n = n; a.d = cache->d; a.dtype = dtype; a.cache_dtype = cache->dtype;
    return launch_cache_read(a, (hipStream_t)hip_stream) == hipSuccess ? OBC_OK : OBC_ELAUNCH;
}

}  // extern "C"
