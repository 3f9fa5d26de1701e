// New rows into a paged K/V cache, with the position rotation on the way (paper App. A: the dual cache is refreshed at block
// boundaries; a paged cache has no counterpart there).
//
// A block takes a row, or several where a row has few heads.  A row's angles, position x inverse frequency, are taken once for all heads: reduced in
// fp64 to an eighth of a turn around the nearest quarter (a position of 10^6 leaves 1e-10 of an angle there; in fp32 it would leave 0.1),
// then sine and cosine in fp32, left in shared memory.  Every thread moves units of 16 dimensions of a head: the two chunks of 8 that
// rotate into each other, or 16 neighbours.  The loads of a batch of units are issued before the angles and the page are looked up.
// Bound by memory: each row is read once and written once, and nothing but the tables comes on top.
#include <cuda_fp8.h>
#include <algorithm>
#include "tsd_paged.cuh"

namespace tsd {

int check_paged_cache(const tsd_paged_cache* c) {
  if (!c || !c->k_pages || !c->v_pages || !c->page_table) return TSD_ERR_INVALID_ARG;
  if (c->batch < 1 || c->n_pages < 1 || c->max_pages < 1 || c->n_kv_heads < 1 || c->table_stride < 0) return TSD_ERR_INVALID_ARG;
  if (c->page_size < 1) return TSD_ERR_INVALID_ARG;
  if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return TSD_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_size > 0x7fffffffll) return TSD_ERR_INVALID_ARG;
  if (c->batch > 1 && c->table_stride < c->max_pages) return TSD_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return TSD_ERR_UNSUPPORTED;
  if (c->dtype != TSD_F32 && c->dtype != TSD_BF16 && c->dtype != TSD_E4M3) return TSD_ERR_UNSUPPORTED;
  if (c->dtype != TSD_E4M3 && (c->k_scale || c->v_scale)) return TSD_ERR_INVALID_ARG;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return TSD_ERR_INVALID_ARG;
  const int esize = c->dtype == TSD_F32 ? 4 : c->dtype == TSD_BF16 ? 2 : 1;
  const int32_t counts[3] = {c->n_pages, c->page_size, c->n_kv_heads};
  for (int i = 0; i < 3; ++i)
    if (counts[i] > 1 && (c->page_stride[i] < c->head_dim || (c->page_stride[i] * esize) % 16 != 0)) return TSD_ERR_INVALID_ARG;
  return TSD_OK;
}

PagedView paged_view(const tsd_paged_cache& c) {
  PagedView v;
  v.k = c.k_pages; v.v = c.v_pages;
  v.ps_p = c.page_stride[0]; v.ps_r = c.page_stride[1]; v.ps_h = c.page_stride[2];
  v.k_scale = c.k_scale; v.v_scale = c.v_scale;
  v.table = c.page_table;
  v.table_stride = c.table_stride;
  v.n_pages = c.n_pages;
  v.shift = 0;
  while ((1 << v.shift) < c.page_size) ++v.shift;
  v.cap = c.max_pages * c.page_size;
  return v;
}

constexpr int kAppendThreads = 256;
constexpr int kAppendUnits = 3;   // units of a thread in flight: a row of 32 heads each of queries, keys and values is one batch
constexpr int kAppendBlocks = 4;  // per SM
constexpr int kAppendRows = 8;    // rows of a block at most

struct AppendParams {
  PagedView cache;
  bool cached;
  int rows, rows_per_block;       // of all sequences
  int n_blocks, n_rows, Hq, Hkv;  // Hq = 0: no queries
  const int32_t *block, *n_new, *first_slot, *positions;
  const float* inv_freq;
  int rot;
  int64_t kv_b, kv_r, kv_h, q_b, q_r, q_h, ko_b, ko_r, ko_h, qo_b, qo_r, qo_h;
  uint32_t* status;
};

struct alignas(16) Chunk8F { float4 a, b; };
// 8 consecutive elements of a row <-> fp32.  Plain loads: a result may go where its input was.
__device__ __forceinline__ Chunk8F load_chunk(const float* p) {
  return {reinterpret_cast<const float4*>(p)[0], reinterpret_cast<const float4*>(p)[1]};
}
__device__ __forceinline__ uint4 load_chunk(const __nv_bfloat16* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void widen(const Chunk8F& c, float (&x)[8]) {
  x[0] = c.a.x; x[1] = c.a.y; x[2] = c.a.z; x[3] = c.a.w;
  x[4] = c.b.x; x[5] = c.b.y; x[6] = c.b.z; x[7] = c.b.w;
}
__device__ __forceinline__ void widen(const uint4& c, float (&x)[8]) {
  const uint32_t u[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store_chunk(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store_chunk(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}
// into a page: the model's type, or e4m3 of x times the scale's reciprocal (an ulp of fp32 beside x / scale; eight divisions a chunk
// would be more work than all the rest)
__device__ __forceinline__ void store_cached(float* p, const float (&x)[8], float) { store_chunk(p, x); }
__device__ __forceinline__ void store_cached(__nv_bfloat16* p, const float (&x)[8], float) { store_chunk(p, x); }
__device__ __forceinline__ void store_cached(uint8_t* p, const float (&x)[8], float unit) {
  uint32_t u[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i] * unit, x[4 * i + 1] * unit), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2] * unit, x[4 * i + 3] * unit), __NV_SATFINITE, __NV_E4M3);
    u[i] = lo | hi << 16;
  }
  *reinterpret_cast<uint2*>(p) = make_uint2(u[0], u[1]);
}

// cos and sin of position * inv_freq.  t = the angle in turns; q = its nearest quarter; the rest, at most an eighth of a turn, is
// small enough that fp32 holds it to 5e-8 of a radian.
__device__ __forceinline__ float2 cos_sin(int position, float inv_freq) {
  const double t = (double)position * (double)inv_freq * 0.15915494309189533577;
  const double quarter = rint(t * 4.0);
  const float rest = (float)fma(quarter, -0.25, t);
  float s, c;
  sincospif(2.f * rest, &s, &c);
  // quarter modulo 4, also of counts beyond 32 bits (an inverse frequency is any float)
  const int turn = (int)(quarter - 4.0 * floor(quarter * 0.25));
  const float cx = turn & 1 ? s : c, sx = turn & 1 ? c : s;
  return make_float2(turn == 1 || turn == 2 ? -cx : cx, turn >= 2 ? -sx : sx);
}

// kNext: neighbouring dimensions (2j, 2j + 1) form the pairs.  kOne: one row per block; every thread looks up by itself whose it is, without a barrier.
template <typename T, typename C, int D, bool kNext, bool kOne>
__global__ void __launch_bounds__(kAppendThreads, kAppendBlocks)
append_kernel(const T* k, const T* v, const T* q, T* k_out, T* q_out, AppendParams p) {
  struct Row {
    int s, from, slot;  // sequence, row of k, v and q (-1: does not count, -2: its block does not exist), slot in the cache
    bool in_cache;      // it is one
  };
  constexpr int kRows = kOne ? 1 : kAppendRows;
  __shared__ float2 turns[kRows][D / 2];
  __shared__ Row rows[kRows];
  __shared__ int64_t row_at[kRows];  // where the row's page has it, in elements; -1: nowhere
  grid_wait(k, v, q, k_out, q_out);
  settle(p.block, p.n_new, p.first_slot, p.positions, p.inv_freq, p.cache.table, p.cache.k_scale, p.cache.v_scale);
  const int tid = threadIdx.x, first = (int)blockIdx.x * (kOne ? 1 : p.rows_per_block), count = kOne ? 1 : min(p.rows_per_block, p.rows - first);
  auto look_up = [&](int f) {
    const int s = (int)((unsigned)f / (unsigned)p.n_rows), i = f - s * p.n_rows;
    const int n_new = p.n_new ? p.n_new[s] : p.n_rows, block = p.block ? p.block[s] : 0;
    const int64_t slot = (int64_t)(p.first_slot ? p.first_slot[s] : 0) + i;
    const bool there = block >= 0 && block < p.n_blocks;
    return Row{s, i >= n_new ? -1 : there ? block * p.n_rows + i : -2, (int)slot, slot >= 0 && slot < p.cache.cap};
  };
  Row only;
  if (kOne) {
    only = look_up(first);
    if (only.from == -1) return;
  } else {
    if (tid < count) rows[tid] = look_up(first + tid);
    __syncthreads();
  }
  auto row_of = [&](int r) -> const Row& { return kOne ? only : rows[r]; };

  // Units of 16 dimensions: heads of q, then of k, then of v, row by row; D / 16 per head.  A thread's units have the same place in their heads.
  constexpr int kPer = D / 16, kStep = kAppendThreads / kPer;
  static_assert(kAppendThreads % kPer == 0, "a thread's place in a head stays the same");
  const int place = tid % kPer, half = p.rot / 2;
  const bool turning = place * 16 < p.rot;
  // the unit's two chunks of 8: dimensions [d0, d0 + 8) and [d1, d1 + 8)
  const int d0_rot = kNext || !turning ? place * 16 : place * 8, d1_rot = kNext || !turning ? place * 16 + 8 : half + place * 8;
  const int heads = p.Hq + p.Hkv + (p.cached ? p.Hkv : 0);
  int row = 0, head = tid / kPer;  // of the thread's next unit
  bool waited = false;
  do {
    decltype(load_chunk(k)) raw[kAppendUnits][2];
    int row0 = row, head0 = head;
#pragma unroll
    for (int u = 0; u < kAppendUnits; ++u, head += kStep) {
      while (head >= heads && row < count) { head -= heads; ++row; }
      if (row >= count || row_of(row).from < 0) continue;
      const int64_t s = row_of(row).s, from = row_of(row).from;
      const T* src = head < p.Hq ? q + s * p.q_b + from * p.q_r + head * p.q_h
                                 : (head < p.Hq + p.Hkv ? k + (head - p.Hq) * p.kv_h : v + (head - p.Hq - p.Hkv) * p.kv_h) + s * p.kv_b + from * p.kv_r;
      const bool is_v = head >= p.Hq + p.Hkv;  // values do not turn
      raw[u][0] = load_chunk(src + (is_v ? place * 16 : d0_rot));
      raw[u][1] = load_chunk(src + (is_v ? place * 16 + 8 : d1_rot));
    }
    if (!waited) {
      for (int e = tid; e < count * half; e += kAppendThreads) {
        const int r = kOne ? 0 : (int)((unsigned)e / (unsigned)half), j = e - r * half, f = first + r;
        if (row_of(r).from >= 0) turns[r][j] = cos_sin(p.positions ? p.positions[f] : row_of(r).slot, p.inv_freq[j]);
      }
      if (tid < count) {
        int64_t at = -1;
        const Row& mine = row_of(tid);
        bool missing = mine.from == -2;
        if (p.cached && mine.from >= 0) {
          const int page = mine.in_cache ? page_of(p.cache, mine.s, mine.slot) : -1;
          if (page >= 0) at = (int64_t)page * p.cache.ps_p + (mine.slot & ((1 << p.cache.shift) - 1)) * p.cache.ps_r;
          else missing = true;
        }
        if (missing && p.status) atomicOr(p.status, TSD_STATUS_BAD_INDEX);
        row_at[tid] = at;
      }
      __syncthreads();
      waited = true;
    }
#pragma unroll
    for (int u = 0; u < kAppendUnits; ++u, head0 += kStep) {
      while (head0 >= heads && row0 < count) { head0 -= heads; ++row0; }
      if (row0 >= count || row_of(row0).from < 0) continue;
      float x[8], y[8];
      widen(raw[u][0], x);
      widen(raw[u][1], y);
      const bool is_v = head0 >= p.Hq + p.Hkv;
      const int d0 = is_v ? place * 16 : d0_rot, d1 = is_v ? place * 16 + 8 : d1_rot;
      if (turning && !is_v) {
        const float2* turn = turns[row0] + place * 8;
        if (kNext) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 a = turn[j], b = turn[4 + j];
            const float x0 = x[2 * j], x1 = x[2 * j + 1], y0 = y[2 * j], y1 = y[2 * j + 1];
            x[2 * j] = x0 * a.x - x1 * a.y;
            x[2 * j + 1] = x0 * a.y + x1 * a.x;
            y[2 * j] = y0 * b.x - y1 * b.y;
            y[2 * j + 1] = y0 * b.y + y1 * b.x;
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 a = turn[j];
            const float x0 = x[j], y0 = y[j];
            x[j] = x0 * a.x - y0 * a.y;
            y[j] = x0 * a.y + y0 * a.x;
          }
        }
      }
      const int64_t s = row_of(row0).s, from = row_of(row0).from;
      if (head0 < p.Hq) {
        T* dst = q_out + s * p.qo_b + from * p.qo_r + head0 * p.qo_h;
        store_chunk(dst + d0, x);
        store_chunk(dst + d1, y);
        continue;
      }
      const int g = head0 - p.Hq - (is_v ? p.Hkv : 0);
      if (!is_v && k_out) {
        T* dst = k_out + s * p.ko_b + from * p.ko_r + g * p.ko_h;
        store_chunk(dst + d0, x);
        store_chunk(dst + d1, y);
      }
      const int64_t at = row_at[row0];
      if (at >= 0) {
        const float* scales = is_v ? p.cache.v_scale : p.cache.k_scale;
        const float unit = sizeof(C) == 1 && scales ? 1.f / scales[g] : 1.f;
        C* dst = const_cast<C*>(static_cast<const C*>(is_v ? p.cache.v : p.cache.k)) + at + g * p.cache.ps_h;
        store_cached(dst + d0, x, unit);
        store_cached(dst + d1, y, unit);
      }
    }
  } while (row < count);
}

template <typename T, typename C, int D>
static cudaError_t launch_append(const tsd_append_args& a, const AppendParams& p, cudaStream_t stream) {
  const bool one = p.rows_per_block == 1;
  const auto kernel = a.interleaved ? (one ? append_kernel<T, C, D, true, true> : append_kernel<T, C, D, true, false>)
                                    : (one ? append_kernel<T, C, D, false, true> : append_kernel<T, C, D, false, false>);
  return launch(kernel, dim3((unsigned)((p.rows + p.rows_per_block - 1) / p.rows_per_block)), dim3(kAppendThreads), 0, stream,
                static_cast<const T*>(a.k), static_cast<const T*>(a.v), static_cast<const T*>(a.q), static_cast<T*>(a.k_out),
                static_cast<T*>(a.q_out), p);
}
template <typename T, typename C>
static cudaError_t launch_append(const tsd_append_args& a, const AppendParams& p, cudaStream_t stream) {
  return a.head_dim == 64 ? launch_append<T, C, 64>(a, p, stream) : launch_append<T, C, 128>(a, p, stream);
}

// Strides (batch, row, head) of rows of heads; a dimension of size 1 may have any.
static bool strides_ok(const int64_t (&st)[3], int batch, int64_t rows, int heads, int head_dim, int esize) {
  const int64_t counts[3] = {batch, rows, heads}, least[3] = {0, 0, head_dim};
  for (int i = 0; i < 3; ++i)
    if (counts[i] > 1 && (st[i] < least[i] || (st[i] * esize) % 16 != 0)) return false;
  return true;
}

static int check_append(const tsd_append_args& a) {
  if (a.batch < 0 || a.n_blocks < 1 || a.n_rows < 0 || a.n_kv_heads < 1 || a.n_q_heads < 0) return TSD_ERR_INVALID_ARG;
  if (a.head_dim != 64 && a.head_dim != 128) return TSD_ERR_UNSUPPORTED;
  if (a.dtype != TSD_F32 && a.dtype != TSD_BF16) return TSD_ERR_UNSUPPORTED;
  if (a.rotary_dim < 0 || a.rotary_dim > a.head_dim || (a.rotary_dim > 0 && !a.inv_freq)) return TSD_ERR_INVALID_ARG;
  if (a.rotary_dim % 16 != 0) return TSD_ERR_UNSUPPORTED;
  if (a.cache) {
    const int rc = check_paged_cache(a.cache);
    if (rc != TSD_OK) return rc;
    if (a.cache->batch != a.batch || a.cache->n_kv_heads != a.n_kv_heads || a.cache->head_dim != a.head_dim) return TSD_ERR_INVALID_ARG;
    if (a.cache->dtype != a.dtype && !(a.cache->dtype == TSD_E4M3 && a.dtype == TSD_BF16)) return TSD_ERR_UNSUPPORTED;
  }
  if (!a.k || (a.cache && !a.v) || (a.q == nullptr) != (a.q_out == nullptr)) return TSD_ERR_INVALID_ARG;
  if (a.q && a.n_q_heads < 1) return TSD_ERR_INVALID_ARG;
  const void* ptrs[] = {a.k, a.v, a.q, a.k_out, a.q_out};
  for (const void* ptr : ptrs)
    if (ptr && !aligned16(ptr)) return TSD_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)a.n_blocks * a.n_rows;
  const int esize = a.dtype == TSD_F32 ? 4 : 2;
  if (!strides_ok(a.kv_stride, a.batch, rows, a.n_kv_heads, a.head_dim, esize)) return TSD_ERR_INVALID_ARG;
  if (a.k_out && !strides_ok(a.k_out_stride, a.batch, rows, a.n_kv_heads, a.head_dim, esize)) return TSD_ERR_INVALID_ARG;
  if (a.q && (!strides_ok(a.q_stride, a.batch, rows, a.n_q_heads, a.head_dim, esize) ||
              !strides_ok(a.q_out_stride, a.batch, rows, a.n_q_heads, a.head_dim, esize)))
    return TSD_ERR_INVALID_ARG;
  if (a.n_q_heads > (1 << 20) || a.n_kv_heads > (1 << 20) || (int64_t)a.batch * a.n_rows > 0x7fffffffll || rows > 0x7fffffffll)
    return TSD_ERR_UNSUPPORTED;
  return TSD_OK;
}

}  // namespace tsd

extern "C" int tsd_append_paged_kv(const tsd_append_args* args, tsd_stream_t stream) {
  if (!args) return TSD_ERR_INVALID_ARG;
  const tsd_append_args& a = *args;
  const int rc = tsd::check_append(a);
  if (rc != TSD_OK || a.batch == 0 || a.n_rows == 0) return rc;
  tsd::AppendParams p = {};
  p.cached = a.cache != nullptr;
  if (p.cached) p.cache = tsd::paged_view(*a.cache);
  p.n_blocks = a.n_blocks; p.n_rows = a.n_rows;
  p.rows = a.batch * a.n_rows;
  p.Hq = a.q ? a.n_q_heads : 0; p.Hkv = a.n_kv_heads;
  p.block = a.block; p.n_new = a.n_new; p.first_slot = a.first_slot; p.positions = a.positions;
  p.inv_freq = a.inv_freq;
  p.rot = a.rotary_dim;
  // as many rows to a block as make one batch of units, if that leaves every SM its four blocks
  const int units = (p.Hq + p.Hkv * (p.cached ? 2 : 1)) * (a.head_dim / 16);
  p.rows_per_block = std::max(1, std::min({tsd::kAppendRows, tsd::kAppendThreads * tsd::kAppendUnits / units, p.rows / (tsd::kAppendBlocks * tsd::kPlanSms)}));
  p.kv_b = a.kv_stride[0]; p.kv_r = a.kv_stride[1]; p.kv_h = a.kv_stride[2];
  p.q_b = a.q_stride[0]; p.q_r = a.q_stride[1]; p.q_h = a.q_stride[2];
  p.ko_b = a.k_out_stride[0]; p.ko_r = a.k_out_stride[1]; p.ko_h = a.k_out_stride[2];
  p.qo_b = a.q_out_stride[0]; p.qo_r = a.q_out_stride[1]; p.qo_h = a.q_out_stride[2];
  p.status = a.status;
  const cudaError_t e = a.dtype == TSD_F32 ? tsd::launch_append<float, float>(a, p, stream)
                        : p.cached && a.cache->dtype == TSD_E4M3 ? tsd::launch_append<__nv_bfloat16, uint8_t>(a, p, stream)
                                                                 : tsd::launch_append<__nv_bfloat16, __nv_bfloat16>(a, p, stream);
  if (e != cudaSuccess) return tsd::cuda_fail(e, "append_kernel");
  return TSD_OK;
}
