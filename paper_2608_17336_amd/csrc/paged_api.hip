// paged_api.hip -- the C ABI of the paged key/value cache: argument checks and launches.
#include <math.h>

#include "tilemix.h"
#include "tilemix_internal.h"

namespace {

using tilemix::api::fail;
using tilemix::api::ok;

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

tilemix_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(TILEMIX_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool is_8bit(int32_t format) { return format == TILEMIX_INT8 || format == TILEMIX_E4M3; }

constexpr long long kStrideMax = 1LL << 40;
// Packed rows, and elements of them: a launch has at most 2^23 workgroups of 256 threads, and one more for each sequence.
constexpr int32_t kRowsMax = 1 << 28;
constexpr long long kRowElementsMax = 1LL << 34;

// Sizes, strides and formats of the pool and its sequences (no pointers).
tilemix_status check_shape(const tilemix_paged_cache* c) {
  if (!c) return fail(TILEMIX_ERR_NULL, "cache is NULL");
  if (c->format < TILEMIX_FP16 || c->format > TILEMIX_E4M3)
    return fail(TILEMIX_ERR_UNSUPPORTED, "cache format %d not supported", c->format);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(TILEMIX_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", c->head_dim);
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return fail(TILEMIX_ERR_UNSUPPORTED, "page_size %d not supported (16, 32, 64, 128 or 256)", c->page_size);
  if (c->pages < 1 || c->heads_kv < 1 || c->batch < 1 || c->max_pages < 1)
    return fail(TILEMIX_ERR_SHAPE, "pages, heads_kv, batch and max_pages must be >= 1");
  if (c->heads_kv > 65535 || c->batch > 65535) return fail(TILEMIX_ERR_SHAPE, "heads_kv and batch must be <= 65535");
  if ((long long)c->max_pages * c->page_size > (1LL << 30))
    return fail(TILEMIX_ERR_SHAPE, "max_pages * page_size must be <= 2^30");
  if (c->stride_table < c->max_pages || c->stride_table > kStrideMax)
    return fail(TILEMIX_ERR_SHAPE, "stride_table must be >= max_pages");
  const long long rows = (long long)c->heads_kv * c->page_size;
  for (long long s : {(long long)c->stride_k, (long long)c->stride_v})
    if (s < rows * c->head_dim || s > kStrideMax || s % 16)
      return fail(TILEMIX_ERR_SHAPE, "page strides must be >= heads_kv * page_size * head_dim and multiples of 16");
  if (is_8bit(c->format))
    for (long long s : {(long long)c->stride_dk, (long long)c->stride_dv})
      if (s < rows || s > kStrideMax || s % 4)
        return fail(TILEMIX_ERR_SHAPE, "scale page strides must be >= heads_kv * page_size and multiples of 4");
  return TILEMIX_OK;
}

tilemix_status check_pointers(const tilemix_paged_cache* c) {
  if (!c->K || !c->V || !c->page_table || !c->seqlens_k)
    return fail(TILEMIX_ERR_NULL, "K, V, page_table and seqlens_k must be non-NULL");
  if (!aligned(c->K, 16) || !aligned(c->V, 16)) return fail(TILEMIX_ERR_ALIGN, "K and V must be 16-byte aligned");
  if (!aligned(c->page_table, 4) || !aligned(c->seqlens_k, 4))
    return fail(TILEMIX_ERR_ALIGN, "page_table and seqlens_k must be 4-byte aligned");
  if (is_8bit(c->format)) {
    if (!c->dK || !c->dV) return fail(TILEMIX_ERR_NULL, "an 8-bit cache needs dK and dV");
    if (!aligned(c->dK, 16) || !aligned(c->dV, 16)) return fail(TILEMIX_ERR_ALIGN, "dK and dV must be 16-byte aligned");
  }
  return TILEMIX_OK;
}

tilemix_status check_type(const tilemix_paged_cache* c, int32_t type) {
  if (type != TILEMIX_FP16 && type != TILEMIX_BF16)
    return fail(TILEMIX_ERR_UNSUPPORTED, "type %d not supported (FP16 or BF16)", type);
  if (!is_8bit(c->format) && type != c->format)
    return fail(TILEMIX_ERR_UNSUPPORTED, "a 16-bit cache takes rows of its own type only");
  return TILEMIX_OK;
}

tilemix::PagedPool pool_of(const tilemix_paged_cache* c) {
  tilemix::PagedPool p{};
  p.K = c->K; p.V = c->V;
  if (is_8bit(c->format)) {
    p.dK = c->dK; p.dV = c->dV;
    p.stride_dk = c->stride_dk; p.stride_dv = c->stride_dv;
  }
  p.table = c->page_table; p.seqlens = c->seqlens_k;
  p.stride_k = c->stride_k; p.stride_v = c->stride_v; p.stride_table = c->stride_table;
  p.pages = c->pages;
  while ((1 << p.page_shift) < c->page_size) ++p.page_shift;
  p.Hk = c->heads_kv; p.B = c->batch; p.max_pages = c->max_pages;
  return p;
}

// What append and gather share; rows: their packed side.  total = 0: *nothing is set.
tilemix_status rows_args(const tilemix_paged_cache* c, int32_t type, const int32_t* cu, int32_t len, int32_t total,
                         const void* K, int64_t k_stride, const void* V, int64_t v_stride,
                         tilemix::PagedRowsArgs* a, bool* nothing) {
  tilemix_status st = check_shape(c);
  if (st != TILEMIX_OK) return st;
  if ((st = check_type(c, type)) != TILEMIX_OK) return st;
  const bool none = cu && total == 0;   // no sequence has a row: the longest has 0
  if (len < (none ? 0 : 1) || len > kRowsMax) return fail(TILEMIX_ERR_SHAPE, "len must be 1 .. %d", kRowsMax);
  if (total < 0 || total > kRowsMax) return fail(TILEMIX_ERR_SHAPE, "total must be 0 .. %d", kRowsMax);
  if ((long long)total * c->heads_kv * c->head_dim > kRowElementsMax)
    return fail(TILEMIX_ERR_SHAPE, "total * heads_kv * head_dim must be <= 2^34");
  if (!cu && total != (long long)c->batch * len) return fail(TILEMIX_ERR_SHAPE, "total must be batch * len without cu_seqlens");
  if (k_stride < 0 || v_stride < 0 || k_stride > kStrideMax || v_stride > kStrideMax || k_stride % 8 || v_stride % 8)
    return fail(TILEMIX_ERR_SHAPE, "row strides must be >= 0 and multiples of 8");
  *nothing = total == 0;
  if (*nothing) return TILEMIX_OK;
  if ((st = check_pointers(c)) != TILEMIX_OK) return st;
  if (!K || !V) return fail(TILEMIX_ERR_NULL, "the rows of K and V must be non-NULL");
  if (!aligned(K, 16) || !aligned(V, 16)) return fail(TILEMIX_ERR_ALIGN, "the rows of K and V must be 16-byte aligned");
  if (cu && !aligned(cu, 4)) return fail(TILEMIX_ERR_ALIGN, "cu_seqlens must be 4-byte aligned");
  a->pool = pool_of(c);
  a->cu = cu; a->len = len; a->total = total;
  a->K = const_cast<void*>(K); a->V = const_cast<void*>(V);
  a->k_stride = k_stride; a->v_stride = v_stride;
  return TILEMIX_OK;
}

tilemix_status check_decode(const tilemix_paged_cache* c, int32_t heads_q) {
  tilemix_status st = check_shape(c);
  if (st != TILEMIX_OK) return st;
  if (heads_q < 1 || heads_q > 65535 || heads_q % c->heads_kv != 0)
    return fail(TILEMIX_ERR_SHAPE, "heads_q (%d) must be a multiple of heads_kv (%d), at most 65535", heads_q, c->heads_kv);
  if (tilemix::plan_paged_decode(pool_of(c), heads_q, c->head_dim, 0).units > (1LL << 30))
    return fail(TILEMIX_ERR_SHAPE, "batch * heads * max_pages * page_size is too large");
  return TILEMIX_OK;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Workspace: [segments][part_mzx][part_o], each 256-byte aligned.
struct DecodeBytes {
  size_t segments, mzx, o;
  size_t total() const { return segments + mzx + o; }
};
DecodeBytes decode_bytes(const tilemix_paged_cache* c, const tilemix::PagedDecodePlan& pl) {
  if (pl.whole) return {0, 0, 0};
  const size_t rows = 2 * (size_t)pl.workgroups * pl.part_heads;
  return {align256((size_t)c->batch * pl.head_blocks * 2 * sizeof(int)), align256(rows * 4 * sizeof(float)),
          align256(rows * c->head_dim * sizeof(float))};
}

}  // namespace

extern "C" {

tilemix_status tilemix_paged_append(const tilemix_paged_cache* cache, int32_t type,
                                    const int32_t* cu_seqlens, int32_t len, int32_t total,
                                    const void* K_new, int64_t k_stride, const void* V_new,
                                    int64_t v_stride, void* stream) {
  tilemix::PagedRowsArgs a{};
  bool nothing;
  const tilemix_status st = rows_args(cache, type, cu_seqlens, len, total, K_new, k_stride, V_new, v_stride, &a, &nothing);
  if (st != TILEMIX_OK) return st;
  if (nothing) return ok();
  return hip_status(tilemix::launch_paged_append(a, cache->head_dim, type, cache->format, static_cast<hipStream_t>(stream)),
                    "paged append");
}

tilemix_status tilemix_paged_gather(const tilemix_paged_cache* cache, int32_t type,
                                    const int32_t* cu_seqlens, int32_t len, int32_t total,
                                    void* K_out, void* V_out, void* stream) {
  tilemix::PagedRowsArgs a{};
  bool nothing;
  const int64_t row = cache ? (int64_t)cache->heads_kv * cache->head_dim : 0;
  const tilemix_status st = rows_args(cache, type, cu_seqlens, len, total, K_out, row, V_out, row, &a, &nothing);
  if (st != TILEMIX_OK) return st;
  if (nothing) return ok();
  return hip_status(tilemix::launch_paged_gather(a, cache->head_dim, type, cache->format, static_cast<hipStream_t>(stream)),
                    "paged gather");
}

tilemix_status tilemix_paged_decode_workspace_size(const tilemix_paged_cache* cache, int32_t heads_q, size_t* bytes) {
  const tilemix_status st = check_decode(cache, heads_q);
  if (st != TILEMIX_OK) return st;
  if (!bytes) return fail(TILEMIX_ERR_NULL, "bytes is NULL");
  *bytes = decode_bytes(cache, tilemix::plan_paged_decode(pool_of(cache), heads_q, cache->head_dim, 0)).total();
  return ok();
}

tilemix_status tilemix_paged_decode(const tilemix_paged_cache* cache, int32_t type, int32_t heads_q, float scale,
                                    int32_t window, const void* Q, int64_t q_stride, void* O, float* lse,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  tilemix_status st = check_decode(cache, heads_q);
  if (st != TILEMIX_OK) return st;
  if ((st = check_type(cache, type)) != TILEMIX_OK) return st;
  if (!(isfinite(scale) && scale > 0.0f)) return fail(TILEMIX_ERR_SHAPE, "scale must be finite and > 0");
  if (window < 0) return fail(TILEMIX_ERR_SHAPE, "window must be >= 0");
  if (q_stride < 0 || q_stride > kStrideMax || q_stride % 8) return fail(TILEMIX_ERR_SHAPE, "q_stride must be >= 0 and a multiple of 8");
  if ((st = check_pointers(cache)) != TILEMIX_OK) return st;
  if (!Q || !O) return fail(TILEMIX_ERR_NULL, "Q and O must be non-NULL");
  if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(lse, 4))
    return fail(TILEMIX_ERR_ALIGN, "Q and O must be 16-byte and lse 4-byte aligned");
  tilemix::PagedDecodeArgs a{};
  a.pool = pool_of(cache);
  const tilemix::PagedDecodePlan pl = tilemix::plan_paged_decode(a.pool, heads_q, cache->head_dim, window);
  const DecodeBytes need = decode_bytes(cache, pl);
  if (need.total()) {
    if (!workspace) return fail(TILEMIX_ERR_WORKSPACE, "workspace is NULL");
    if (!aligned(workspace, 256)) return fail(TILEMIX_ERR_ALIGN, "workspace must be 256-byte aligned");
    if (workspace_bytes < need.total())
      return fail(TILEMIX_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need.total());
    char* ws = static_cast<char*>(workspace);
    a.segments = reinterpret_cast<int*>(ws);
    a.part_mzx = reinterpret_cast<float*>(ws + need.segments);
    a.part_o = reinterpret_cast<float*>(ws + need.segments + need.mzx);
  }
  a.head_blocks = pl.head_blocks;
  a.whole = pl.whole;
  a.part_heads = pl.part_heads;
  a.Q = Q; a.O = O; a.lse = lse; a.q_stride = q_stride;
  a.Hq = heads_q; a.window = window;
  a.scale_log2e = scale * 1.4426950408889634f;
  return hip_status(tilemix::launch_paged_decode(a, pl, cache->head_dim, type, cache->format, static_cast<hipStream_t>(stream)),
                    "paged decode");
}

}  // extern "C"
