// New rows into a paged K/V cache, with the position rotation on the way (paper App. A: the dual cache is refreshed at block
// boundaries; a paged cache has no counterpart there).
//
// A warp takes a row, or, with few rows, some heads of one.  It walks them in units of 16 dimensions per lane: two chunks of 8, half a head
// apart, which are those that rotate into each other, and in any case such that an instruction of the warp touches whole
// 128-byte lines.  The next kAppendAhead units, of the rows to come too, are on their way to shared memory (cp.async; a lane reads
// back what it has fetched, so nothing is waited for but the lane's own fetches).  A lane's units all have the same place in their
// heads, so their 8 angles, position x inverse frequency, stay in registers for a row: reduced in fp64 to an eighth of a turn
// around the nearest quarter (a position of 10^6 leaves 1e-10 of an angle there; in fp32 it would leave 0.1), then sine and cosine in
// fp32, two per lane and handed on through shared memory.
// Bound by memory: each row is read once and written once, and nothing but the tables comes on top.  Measured (cold): 16 prompts of 1504 rows,
// 32 heads of 128, q rotated in the same pass: 206 us, 5.7 TB/s, 88 % of what a copy reaches; 1845 rows of 4 heads into e4m3 pages
// and 28 heads of q: 8.6 us, 3.7 TB/s; one row for each of 8 sequences: 3.8 us, of which the launch is most.
#include <cuda_fp8.h>
#include <algorithm>
#include "tsd_paged.cuh"

namespace tsd {

int check_paged_cache(const tsd_paged_cache* c) {
  if (!c || !c->k_pages || !c->v_pages || !c->page_table) return TSD_ERR_INVALID_ARG;
  if (c->batch < 1 || c->n_pages < 1 || c->max_pages < 1 || c->n_kv_heads < 1 || c->table_stride < 0) return TSD_ERR_INVALID_ARG;
  if (c->page_size < 1) return TSD_ERR_INVALID_ARG;
  if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return TSD_ERR_UNSUPPORTED;
  // room behind the last token for the kernels to count on: 32 tiles of 64 keys in the verification pass, whose lanes look up a tile's page each
  if ((int64_t)c->max_pages * c->page_size > 0x80000000ll - 4096) return TSD_ERR_INVALID_ARG;
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

constexpr int kAppendWarps = 8;    // of a block
constexpr int kAppendBlocks = 2;   // per SM
constexpr int kAppendAhead = 5;    // units on their way, of 32 bytes per lane (fp32: half as many, of 64)

struct AppendParams {
  PagedView cache;
  bool cached;
  int S, units, parts;            // units of a row per lane; parts that a row is cut into
  int n_blocks, n_rows, Hq, Hkv;  // Hq = 0: no queries
  const int32_t *block, *n_new, *first_slot, *positions;
  const float* inv_freq;
  int rot;
  int64_t kv_b, kv_r, kv_h, q_b, q_r, q_h, ko_b, ko_r, ko_h, qo_b, qo_r, qo_h;
  uint32_t* status;
};

// 8 consecutive elements <-> fp32.  Ordinary stores: a result may go where its input was.
__device__ __forceinline__ void widen(const uint4* c, float (&x)[8], float) {  // fp32: the second 16 bytes lie one piece of all lanes on
  const float4 a = *reinterpret_cast<const float4*>(c), b = *reinterpret_cast<const float4*>(c + 32);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void widen(const uint4* c, float (&x)[8], __nv_bfloat16) {
  const uint4 v = *c;
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
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
__device__ __forceinline__ float2 cos_sin(int64_t position, float inv_freq) {
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

template <typename T, typename C, int D, bool kNext>  // kNext: neighbouring dimensions (2j, 2j + 1) form the pairs
__global__ void __launch_bounds__(kAppendWarps * 32, kAppendBlocks)
append_kernel(const T* k, const T* v, const T* q, T* k_out, T* q_out, AppendParams p) {
  constexpr int kPer = D / 16, kHeads = 32 / kPer;               // units per head; heads per unit of a warp
  constexpr int kPieces = 2 * (int)sizeof(T) / 2;                // 16-byte pieces of a unit: 2, fp32 4
  constexpr int kAhead = kAppendAhead / (int)(sizeof(T) / 2);
  __shared__ uint4 queue[kAppendWarps][kAhead][kPieces][32];
  __shared__ float2 turns[kAppendWarps][D / 2];
  constexpr unsigned full = 0xffffffffu;
  grid_wait(k, v, q, k_out, q_out);
  settle(p.block, p.n_new, p.first_slot, p.positions, p.inv_freq, p.cache.table, p.cache.k_scale, p.cache.v_scale);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, place = lane % kPer, half = p.rot / 2;
  // A unit's two chunks of 8: dimensions [place * 8, + 8) and [D / 2 + place * 8, + 8).  Halves of rot < D dimensions that rotate into each other
  // are closer: the first rot / 16 places take these, the others 16 neighbours behind them.
  const bool closer = !kNext && p.rot > 0 && p.rot < D, turning = kNext ? place * 8 < p.rot : place * 16 < p.rot;
  // Neighbours: the second chunk lies behind rot before the first one does, and what lies there is copied (times a turn of 0 an infinity
  // would make its neighbour NaN).
  const bool both = D / 2 + place * 8 < p.rot;
  const int d0_rot = closer && !turning ? place * 16 : place * 8, d1_rot = !closer ? D / 2 + place * 8 : turning ? half + place * 8 : place * 16 + 8;
  const int heads = p.Hq + p.Hkv + (p.cached ? p.Hkv : 0);

  // Rows that count, one behind the other (up to 32 sequences; more: all rows, and those that do not count are passed over)
  const bool counted = p.n_new && p.S <= 32;
  int upto = 0, n_rows = p.S * p.n_rows;
  if (counted) {
    const int mine = lane < p.S ? min(max(p.n_new[lane], 0), p.n_rows) : 0;
    upto = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(full, upto, off);
      if (lane >= off) upto += o;
    }
    n_rows = __shfl_sync(full, upto, 31);
  }
  struct Row {
    int s, i;
    int64_t from;  // row of k, v and q; -1: its block does not exist
  };
  auto row_at = [&](int r) {
    Row row;
    if (counted) {
      row.s = __ffs(__ballot_sync(full, upto > r)) - 1;
      row.i = r - (row.s > 0 ? __shfl_sync(full, upto, row.s - 1) : 0);
    } else {
      row.s = (int)((unsigned)r / (unsigned)p.n_rows);
      row.i = r - row.s * p.n_rows;
    }
    const int block = p.block ? p.block[row.s] : 0;
    row.from = block >= 0 && block < p.n_blocks ? (int64_t)block * p.n_rows + row.i : -1;
    return row;
  };
  // A task is a part of a row: units [first, last).  The warps take the tasks in turn.
  const int n_tasks = n_rows * p.parts, stride = (int)gridDim.x * kAppendWarps;  // fewer than 2^31: checked on the host
  struct Task {
    int t, unit, last;
    Row row;
  };
  auto next_task = [&](int t) {  // the task from t on, in strides, whose row counts; t >= n_tasks: none
    Task k;
    for (;; t += stride) {
      k.t = t;
      k.unit = k.last = 0;
      if (t >= n_tasks) return k;
      const int r = p.parts == 1 ? t : (int)((unsigned)t / (unsigned)p.parts), part = t - r * p.parts;
      k.row = row_at(r);
      if (!counted && p.n_new && k.row.i >= p.n_new[k.row.s]) continue;
      if (k.row.from < 0) {
        if (lane == 0 && p.status) atomicOr(p.status, TSD_STATUS_BAD_INDEX);
        continue;
      }
      k.unit = p.parts == 1 ? 0 : (int)((unsigned)(part * p.units) / (unsigned)p.parts);
      k.last = p.parts == 1 ? p.units : (int)((unsigned)((part + 1) * p.units) / (unsigned)p.parts);
      return k;
    }
  };

  // what is fetched, kAhead units before it is needed
  Task ahead = next_task((int)blockIdx.x * kAppendWarps + warp);
  Task task = ahead;
  int slot_in = 0, slot_out = 0;
  const uint32_t queue_at = (uint32_t)__cvta_generic_to_shared(&queue[warp][0][0][lane]);
  // What has been read leaves L2 before what is written, which attention wants next.  (1.2 GB 215 -> 206 us, 1845 rows into e4m3 pages 9.3 -> 8.6;
  // 0.44 GB 72.0 -> 73.4.)
  uint64_t read_once;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(read_once));
  auto fetch = [&] {
    if (ahead.t < n_tasks) {
      const int head = ahead.unit * kHeads + lane / kPer;
      if (head < heads) {
        const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.Hkv;
        const T* src = is_q ? q + ahead.row.s * p.q_b + ahead.row.from * p.q_r + head * p.q_h
                            : (is_v ? v + (head - p.Hq - p.Hkv) * p.kv_h : k + (head - p.Hq) * p.kv_h) + ahead.row.s * p.kv_b + ahead.row.from * p.kv_r;
        const uint32_t to = queue_at + slot_in * (kPieces * 512);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int chunk = i / (kPieces / 2), in = i % (kPieces / 2) * (16 / (int)sizeof(T));
          const T* from = src + (chunk == 0 ? (is_v ? place * 8 : d0_rot) : (is_v ? D / 2 + place * 8 : d1_rot)) + in;
          asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(to + i * 512), "l"(from), "l"(read_once) : "memory");
        }
      }
      if (++ahead.unit == ahead.last) ahead = next_task(ahead.t + stride);
      slot_in = slot_in + 1 == kAhead ? 0 : slot_in + 1;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int i = 0; i < kAhead; ++i) fetch();

#pragma unroll 1
  for (; task.t < n_tasks; task = next_task(task.t + stride)) {
    // where the row goes, and its angles
    const int s = task.row.s;
    const int64_t slot = (int64_t)(p.first_slot ? p.first_slot[s] : 0) + task.row.i, from = task.row.from;
    int64_t at = -1;
    if (p.cached) {
      const int page = slot >= 0 && slot < p.cache.cap ? page_of(p.cache, s, (int)slot) : -1;
      if (page >= 0) at = (int64_t)page * p.cache.ps_p + (slot & ((1 << p.cache.shift) - 1)) * p.cache.ps_r;
      else if (lane == 0 && p.status) atomicOr(p.status, TSD_STATUS_BAD_INDEX);
    }
    float2 turn[8];
    if (half > 0) {
      const int64_t position = p.positions ? p.positions[s * (int64_t)p.n_rows + task.row.i] : slot;
      __syncwarp();
#pragma unroll 1
      for (int j = lane; j < half; j += 32) turns[warp][j] = cos_sin(position, p.inv_freq[j]);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // neighbours: of the first chunk's pairs, then of the second one's
        const int pair = kNext ? (j < 4 ? 0 : D / 4 - 4) + place * 4 + j : place * 8 + j;
        turn[j] = pair < half ? turns[warp][pair] : make_float2(1.f, 0.f);
      }
    }
#pragma unroll 1
    for (int unit = task.unit; unit < task.last; ++unit) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      __syncwarp();
      const int head = unit * kHeads + lane / kPer;
      float x[8], y[8];
      widen(&queue[warp][slot_out][0][lane], x, T());
      widen(&queue[warp][slot_out][kPieces / 2][lane], y, T());
      slot_out = slot_out + 1 == kAhead ? 0 : slot_out + 1;
      fetch();  // into the place of a unit that has been read
      if (head >= heads) continue;
      const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.Hkv;  // values do not turn
      const int d0 = is_v ? place * 8 : d0_rot, d1 = is_v ? D / 2 + place * 8 : d1_rot;
      if (turning && !is_v) {
        if (kNext) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 a = turn[j], b = turn[4 + j];
            const float x0 = x[2 * j], x1 = x[2 * j + 1], y0 = y[2 * j], y1 = y[2 * j + 1];
            x[2 * j] = x0 * a.x - x1 * a.y;
            x[2 * j + 1] = x0 * a.y + x1 * a.x;
            if (both) {
              y[2 * j] = y0 * b.x - y1 * b.y;
              y[2 * j + 1] = y0 * b.y + y1 * b.x;
            }
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
      if (is_q) {
        T* dst = q_out + s * p.qo_b + from * p.qo_r + head * p.qo_h;
        store_chunk(dst + d0, x);
        store_chunk(dst + d1, y);
        continue;
      }
      const int g = head - p.Hq - (is_v ? p.Hkv : 0);
      if (!is_v && k_out) {
        T* dst = k_out + s * p.ko_b + from * p.ko_r + g * p.ko_h;
        store_chunk(dst + d0, x);
        store_chunk(dst + d1, y);
      }
      if (at >= 0) {
        const float* scales = is_v ? p.cache.v_scale : p.cache.k_scale;
        const float unit_scale = sizeof(C) == 1 && scales ? 1.f / scales[g] : 1.f;
        C* dst = const_cast<C*>(static_cast<const C*>(is_v ? p.cache.v : p.cache.k)) + at + g * p.cache.ps_h;
        store_cached(dst + d0, x, unit_scale);
        store_cached(dst + d1, y, unit_scale);
      }
    }
  }
}

template <typename T, typename C, int D>
static cudaError_t launch_append(const tsd_append_args& a, const AppendParams& p, cudaStream_t stream) {
  const int64_t tasks = (int64_t)a.batch * a.n_rows * p.parts;
  const int64_t grid = std::min<int64_t>(kAppendBlocks * kPlanSms, (tasks + kAppendWarps - 1) / kAppendWarps);
  return launch(a.interleaved ? append_kernel<T, C, D, true> : append_kernel<T, C, D, false>, dim3((unsigned)grid), dim3(kAppendWarps * 32), 0, stream,
                static_cast<const T*>(a.k), static_cast<const T*>(a.v), static_cast<const T*>(a.q), static_cast<T*>(a.k_out),
                static_cast<T*>(a.q_out), p);
}
template <typename T, typename C>
static cudaError_t launch_append(const tsd_append_args& a, const AppendParams& p, cudaStream_t stream) {
  return a.head_dim == 64 ? launch_append<T, C, 64>(a, p, stream) : launch_append<T, C, 128>(a, p, stream);
}

// Strides (batch, row, head) of rows of heads; a dimension of size 1 may have any.  What is only read may be the same for all sequences or rows.
static bool strides_ok(const int64_t (&st)[3], int batch, int64_t rows, int heads, int head_dim, int esize, bool written) {
  const int64_t counts[3] = {batch, rows, heads}, each = written ? head_dim : 0, least[3] = {each, each, head_dim};
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
  if (!strides_ok(a.kv_stride, a.batch, rows, a.n_kv_heads, a.head_dim, esize, false)) return TSD_ERR_INVALID_ARG;
  if (a.k_out && !strides_ok(a.k_out_stride, a.batch, rows, a.n_kv_heads, a.head_dim, esize, true)) return TSD_ERR_INVALID_ARG;
  if (a.q && (!strides_ok(a.q_stride, a.batch, rows, a.n_q_heads, a.head_dim, esize, false) ||
              !strides_ok(a.q_out_stride, a.batch, rows, a.n_q_heads, a.head_dim, esize, true)))
    return TSD_ERR_INVALID_ARG;
  if (a.n_q_heads > (1 << 20) || a.n_kv_heads > (1 << 20) || (int64_t)a.batch * a.n_rows > 0x7ff00000ll || rows > 0x7fffffffll)
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
  p.S = a.batch;
  p.Hq = a.q ? a.n_q_heads : 0; p.Hkv = a.n_kv_heads;
  p.block = a.block; p.n_new = a.n_new; p.first_slot = a.first_slot; p.positions = a.positions;
  p.inv_freq = a.inv_freq;
  p.rot = a.rotary_dim;
  // a row is cut where there are fewer rows than warps
  const int per = 32 / (a.head_dim / 16);
  p.units = (p.Hq + p.Hkv * (p.cached ? 2 : 1) + per - 1) / per;
  p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(p.units, tsd::kAppendBlocks * tsd::kPlanSms * tsd::kAppendWarps / ((int64_t)a.batch * a.n_rows)));
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
