// Verify attention (paper Section 3.3) with the cached keys and values in pages.  bf16 pages are read where they are: the tensor-core
// kernel's copies name a page as the outermost coordinate of their tensor maps.  For 8-bit and fp32 pages, and where the
// CUDA-core kernel is asked for, one streaming launch puts the used rows of both caches in order in the workspace (8-bit codes
// as bf16(decode(code) * scale)), and the attention runs on that copy, as it does for a dense 8-bit cache.
// Reading in place costs nothing against a dense cache with pages of 64 rows (4 sequences x 32 branches x 32 rows, 28/4 heads of 128, up to 5056
// cached rows: 213 us, dense 211) and grows with the pages' number (8 rows: 313 us), since a copy of 64 keys is then 8 instructions.
// The ordering of 4 x 1200 rows of 8 e4m3 heads of 64 takes 4.4 us in front of 44 us of attention.  An 8-bit operand read in place
// would have to be widened between its copy and the products, by warps that the softmax needs.
#include <cuda_fp8.h>
#include "tsd_paged.cuh"

namespace tsd {

// 16 elements of a row
__device__ __forceinline__ void move16(const uint8_t* src, float scale, __nv_bfloat16* dst) {
  const uint4 w = *reinterpret_cast<const uint4*>(src);
  const uint32_t words[4] = {w.x, w.y, w.z, w.w};
  uint32_t out[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_fp8x2_storage_t pair = (__nv_fp8x2_storage_t)((words[i >> 1] >> (16 * (i & 1))) & 0xffffu);
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(pair, __NV_E4M3)));  // exact: e4m3 is a subset of fp16
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);
    out[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  reinterpret_cast<uint4*>(dst)[0] = make_uint4(out[0], out[1], out[2], out[3]);
  reinterpret_cast<uint4*>(dst)[1] = make_uint4(out[4], out[5], out[6], out[7]);
}
template <typename T>
__device__ __forceinline__ void move16(const T* src, float, T* dst) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4*>(dst)[i] = reinterpret_cast<const uint4*>(src)[i];
}

// A thread per 16 elements; grid y = sequence, z = K or V.
template <typename C, typename T>
__global__ void __launch_bounds__(256)
order_pages_kernel(PagedView c, const int32_t* __restrict__ mask_blob, T* __restrict__ k_dst, T* __restrict__ v_dst, int Nc, int H, int d,
                   uint32_t vec_per_seq, uint32_t* __restrict__ status) {
  grid_wait(c.k, c.v, c.table, c.k_scale, c.v_scale, mask_blob);
  const uint32_t v = blockIdx.x * blockDim.x + threadIdx.x;
  if (v >= vec_per_seq) return;
  const uint32_t vec_per_head = (uint32_t)d / 16u, vec_per_row = vec_per_head * (uint32_t)H;
  const uint32_t row = v / vec_per_row, cv = v - row * vec_per_row;
  const uint32_t h = cv / vec_per_head, e = cv - h * vec_per_head;
  const int64_t s = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  // Rows at or past the sequence's cache length are not read, and what their places in the copy hold does not matter.
  if ((int)row >= min(max(mask_blob[kHdrWords + s], 0), Nc)) return;
  T* dst = (is_v ? v_dst : k_dst) + (((s * Nc + row) * H + h) * (int64_t)d + e * 16);
  const int page = page_of(c, s, (int)row);
  if (page < 0) {
    for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0, 0, 0, 0);
    if (cv == 0 && !is_v && status) atomicOr(status, TSD_STATUS_BAD_INDEX);
    return;
  }
  const float* scale = is_v ? c.v_scale : c.k_scale;
  const C* src = static_cast<const C*>(is_v ? c.v : c.k) + page * c.ps_p + (row & ((1 << c.shift) - 1)) * c.ps_r + h * c.ps_h + e * 16;
  move16(src, scale ? scale[h] : 1.f, dst);
}

static bool in_place(const tsd_paged_cache& c, uint32_t flags) { return c.dtype == TSD_BF16 && !(flags & TSD_ATTN_FORCE_SIMT); }

static int check_pair(const tsd_layout* L, const tsd_paged_cache* c) {
  int rc = validate_layout(L);
  if (rc == TSD_OK) rc = check_paged_cache(c);
  if (rc != TSD_OK) return rc;
  if (c->batch != L->batch || c->n_kv_heads != L->n_kv_heads || c->head_dim != L->head_dim ||
      (int64_t)c->max_pages * c->page_size < L->n_cache)
    return TSD_ERR_INVALID_ARG;
  if (c->dtype != L->dtype && !(c->dtype == TSD_E4M3 && L->dtype == TSD_BF16)) return TSD_ERR_UNSUPPORTED;
  return TSD_OK;
}

static size_t ordered_bytes(const tsd_layout& L) {
  const size_t bytes = (size_t)L.batch * L.n_cache * L.n_kv_heads * L.head_dim * (L.dtype == TSD_F32 ? 4 : 2);
  return (bytes + 255) / 256 * 256;
}

}  // namespace tsd

extern "C" size_t tsd_verify_attention_paged_workspace_bytes(const tsd_layout* L, const tsd_paged_cache* c, uint32_t flags) {
  if (tsd::check_pair(L, c) != TSD_OK) return 0;
  return tsd::in_place(*c, flags) ? 0 : 2 * tsd::ordered_bytes(*L);
}

extern "C" int tsd_verify_attention_paged(const tsd_layout* L, const void* mask, const void* q, int64_t q_stride_b,
                                          int64_t q_stride_row, int64_t q_stride_head, const tsd_paged_cache* c,
                                          const void* k_draft, const void* v_draft, int64_t d_stride_b,
                                          int64_t d_stride_row, int64_t d_stride_head, void* out, int64_t o_stride_b,
                                          int64_t o_stride_row, int64_t o_stride_head, float* lse, float sm_scale,
                                          void* workspace, size_t workspace_bytes, uint32_t flags, uint32_t* status,
                                          tsd_stream_t stream) {
  int rc = tsd::check_pair(L, c);
  if (rc != TSD_OK) return rc;
  const bool in_place = tsd::in_place(*c, flags);
  const size_t need = tsd_verify_attention_paged_workspace_bytes(L, c, flags);
  if (need > 0 && !workspace) return TSD_ERR_INVALID_ARG;
  if (workspace_bytes < need) return TSD_ERR_WORKSPACE;
  const int64_t hs = L->head_dim, rs = L->n_kv_heads * hs, bs = L->n_cache * rs;
  char* ws = static_cast<char*>(workspace);
  // the cache that the checks of the attention call see: the ordered copy, or (read in place) the pages, checked above
  const void* kc = in_place ? c->k_pages : need ? ws : nullptr;
  const void* vc = in_place ? c->v_pages : need ? ws + need / 2 : nullptr;
  rc = tsd::check_attention_args(L, mask, q, q_stride_b, q_stride_row, q_stride_head, kc, vc, bs, rs, hs, k_draft, v_draft, d_stride_b,
                                 d_stride_row, d_stride_head, out, o_stride_b, o_stride_row, o_stride_head, sm_scale,
                                 need ? workspace : nullptr);
  if (rc != TSD_OK) return rc;
  const tsd::PagedView view = tsd::paged_view(*c);
  tsd::AttnArgs a;
  a.L = *L;
  a.mask = static_cast<const int32_t*>(mask);
  a.q = q; a.kc = kc; a.vc = vc; a.kd = k_draft; a.vd = v_draft; a.out = out; a.lse = lse;
  a.qs_b = q_stride_b; a.qs_r = q_stride_row; a.qs_h = q_stride_head;
  a.cs_b = bs; a.cs_r = rs; a.cs_h = hs;
  a.ds_b = d_stride_b; a.ds_r = d_stride_row; a.ds_h = d_stride_head;
  a.os_b = o_stride_b; a.os_r = o_stride_row; a.os_h = o_stride_head;
  a.sm_scale = sm_scale;
  a.workspace = nullptr;
  a.workspace_bytes = 0;
  a.status = status;
  a.stream = stream;
  a.concurrent = a.next_at_once = false;
  if (in_place && L->n_cache > 0) {
    a.pages = &view;
    return tsd::attention_tc_supported(a) ? tsd::launch_attention_tc(a) : TSD_ERR_UNSUPPORTED;
  }
  if (need > 0) {
    const int64_t vec_per_seq = (int64_t)L->n_cache * L->n_kv_heads * (L->head_dim / 16);
    if (vec_per_seq > 0x7fffff00ll || L->batch > 65535) return TSD_ERR_UNSUPPORTED;  // 32-bit indices, grid y
    const dim3 grid((unsigned)((vec_per_seq + 255) / 256), (unsigned)L->batch, 2);
    cudaError_t e;
    if (c->dtype == TSD_F32)
      e = tsd::launch(tsd::order_pages_kernel<float, float>, grid, 256, 0, stream, view, a.mask, reinterpret_cast<float*>(ws),
                      reinterpret_cast<float*>(ws + need / 2), L->n_cache, L->n_kv_heads, L->head_dim, (uint32_t)vec_per_seq, status);
    else if (c->dtype == TSD_BF16)
      e = tsd::launch(tsd::order_pages_kernel<__nv_bfloat16, __nv_bfloat16>, grid, 256, 0, stream, view, a.mask,
                      reinterpret_cast<__nv_bfloat16*>(ws), reinterpret_cast<__nv_bfloat16*>(ws + need / 2), L->n_cache, L->n_kv_heads,
                      L->head_dim, (uint32_t)vec_per_seq, status);
    else
      e = tsd::launch(tsd::order_pages_kernel<uint8_t, __nv_bfloat16>, grid, 256, 0, stream, view, a.mask,
                      reinterpret_cast<__nv_bfloat16*>(ws), reinterpret_cast<__nv_bfloat16*>(ws + need / 2), L->n_cache, L->n_kv_heads,
                      L->head_dim, (uint32_t)vec_per_seq, status);
    if (e != cudaSuccess) return tsd::cuda_fail(e, "order_pages_kernel");
  }
  return tsd::launch_attention(a, flags);
}
