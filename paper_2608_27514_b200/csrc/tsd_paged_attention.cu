// Attention of one new token per sequence over a paged K/V cache (no counterpart in the paper, whose passes verify whole blocks:
// tsd_verify_attention).  With q the query rows of the heads that share a kv head,
//     s_t = sm_scale <q, k_t>,   out = sum_t e^(s_t - m) v_t / sum_t e^(s_t - m),   m >= max_t s_t - 8 log 2 (8-bit values: - 15).
// Every cached row is read once and used for a few multiply-adds per head, so the kernel is bound by memory; everything in it
// serves to keep loads in flight and the work behind them short.
//   split   : the keys of all sequences and heads are laid end to end in chunks of 4 KB of K and 4 KB of V (16 keys of 128 bf16) and cut over
//             the blocks, one per SM, evenly or item by item (an item: a sequence and a tile of the heads that share one of its kv
//             heads), by the device from the lengths, or, where the caches are short, by the host: a cluster of blocks for every item.  A
//             block's warps take an even stretch of its chunks each, and walk it without waiting for one another.
//   queue   : every warp has its next chunk on the way to shared memory while it works on one (cp.async): 12 warps, 96 KB per SM.  (2
//             sequences of 131072 rows: 12 warps 89.1 us, 16 with fewer registers 92.5, 8 91.4; 64 ragged ones in e4m3: 78.3, 80.7, 85.7.)
//   products: mma.sync m16n8k16 with K (16 keys) or V^T (16 dimensions) as the 16 rows and the heads as the 8 columns: no part of a product is
//             wasted on 8 heads, and O takes 32 registers.  Which dimensions a step of the contraction takes is arbitrary as long as q is
//             laid out alike: lane (g, t) = (lane / 4, lane % 4) reads 16 bytes of keys g and g + 8 at offset 64 c + 16 t, and these bytes
//             are the operand as they are.  For V^T the lane reads columns 8 g ... of keys 2t, 2t+1, 2t+8, 2t+9 and pairs the keys'
//             halves (a byte permutation per register).  Weights go from the one layout to the other by movmatrix, in two
//             16-bit parts (high, residual: off by 2^-17 of the weight; for 8-bit values, f16 parts, by 2^-22 of it and 2^-32 of the largest
//             one).  8-bit codes become f16, one conversion per pair.  The tensor-memory instructions would want 128 rows, and the scores back
//             through tensor memory.
//   offset  : m moves only when a score passes it by 8 (in the exp2 domain; 8-bit values: 15): one vote per chunk instead of a reduction.
//   fp32    : the same queue on CUDA cores (the scores' partial sums of a key meet over its 4 lanes, the weights in shared memory).
//   join    : an item that a warp has from its first chunk to its last is written out at once.  Otherwise the warps' offsets, sums and rows meet
//             in shared memory, and what is not the whole of its item goes to the workspace: the last of the item's blocks to
//             arrive puts the parts together, in their order whoever arrives last, so that results repeat bit by bit.  The blocks
//             of a cluster read one another's parts in shared memory instead.
// Lengths are read on the device: a captured call follows them.  Rows past a length are not loaded.
// Measured (caches larger than L2): 2 sequences of 131072 rows, 28/4 heads of 128, bf16, pages of 64: 84.2 us in runs of 30 calls, 6.4 TB/s, 97 %
// of what a copy reaches (88.6 and 92 % in long runs, at lower clocks); the same in e4m3: 48.4 us, 5.5 TB/s, where conversions come beside the
// loads; 64/4 heads, tiles of 16: 93.4, in e4m3 67.3; 2 of 65536 in fp32, 4/4 heads 87.0 us, 6.2 TB/s, 28/4 heads 142.8, where the query rows'
// loads are the limit; 48 ragged sequences of up to 4096, bf16: 39.9 us, 4.8 TB/s.  A call costs about 6 us before its bytes count (the launch
// and two dependent reads, 2 us; the first chunk on its way, 1 us; the warps' parts, 1 us; the blocks', 2 us), with clusters 4: 1 sequence of 768
// rows, 32 heads (12.6 MB): 6.6 us.
#include <cuda_fp16.h>
#include <algorithm>
#include <cfloat>
#include <math_constants.h>
#include <mutex>
#include "tsd_paged.cuh"

namespace tsd {

constexpr int kTokenBlocks = kPlanSms;  // at most: what the workspace is sized for
constexpr int kAlignSlack = 4;          // the part of a share by which it may grow to keep items apart
constexpr int kReadPast = 4096;         // chunks: 32 MB, a quarter of L2
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;           // by how much a score may pass what the offset was set by, as a power of 2
// How far below the largest score the offset is set, as a power of 2.  The weights of 8-bit values are two f16 parts, and f16 ends at 2^-24:
// with the largest weight at 2^7 or above what is lost of a weight is 2^-32 of that one (at 1, 2^-25: keys 17.5 nats below another were in the
// sum of weights, but not in that of the values).  2^(7 + 8) is still an f16.
template <int kType>
constexpr float kBelow = kType == TSD_E4M3 ? 7.f : 0.f;
constexpr float kLowest = -FLT_MAX;     // the first offset: finite, so that a score of -infinity has the weight 0 from the first key on

enum { kTypeF32 = TSD_F32, kTypeBf16 = TSD_BF16, kTypeE4m3 = TSD_E4M3 };

template <int D, int kType, int HT>  // HT: heads per tile, 8 or 16
struct TokenPlan {
  static constexpr int kWarps = HT == 8 ? 12 : 8;                              // at 168 and 255 registers a thread
  static constexpr int kSize = kType == kTypeF32 ? 4 : kType == kTypeBf16 ? 2 : 1;  // bytes of a cached element
  static constexpr int kRow = D * kSize;                                       // bytes of a row
  static constexpr int kPieces = kRow / 64;                                    // 16-byte pieces per lane and key
  static constexpr int kGroups = 8 / kPieces;                                  // groups of 8 keys per chunk
  static constexpr int kKeys = 8 * kGroups;                                    // keys per chunk
  static constexpr int kSlot = HT * D + 2 * HT;                                // floats of a part in the workspace
  // dynamic shared memory: the warps' queues (a chunk's K, its V), then a part of each warp
  static constexpr int kQueue = kWarps * 8192;
  static constexpr int kPart = HT * D;                                         // floats: at most a warp's queue
  static constexpr int kBytes = kQueue + kWarps * kPart * 4;
  template <bool kItems>
  static constexpr int kBytesFor = kBytes + (kItems ? kSlot * 4 : 0);          // and the block's part, for the others of its cluster
};

struct TokenParams {
  PagedView cache;
  const void* q;
  void* out;
  float* lse;
  const int32_t* lens;
  int64_t q_b, q_h, o_b, o_h;
  int S, Hq, Hkv, group, tiles;  // tiles: of HT heads per kv head
  int shift;                     // 2^shift blocks per item, where the host cuts
  float scale_log2e;
  float* parts;        // [2 * blocks] slots: a block's part of the item that began in a block before it (even), of one that goes on behind it (odd)
  unsigned* tickets;   // per block in which a shared sequence begins
  uint32_t* status;
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// A pair of weights as two 16-bit numbers, and what is left of them.
template <bool kF16>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t& pair, uint32_t& rest) {
  if constexpr (kF16) {
    pair = f16_pair(x, y);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&pair));
    rest = f16_pair(x - f.x, y - f.y);
  } else {
    pair = bf16_pair(x, y);
    rest = bf16_pair(x - __uint_as_float(pair << 16), y - __uint_as_float(pair & 0xffff0000u));
  }
}
// 16 bytes of the cache, or zeros, into shared memory, asynchronously; `policy`: what L2 is to do with their line.
__device__ __forceinline__ void fetch16(uint32_t to, const uint8_t* p, bool wanted, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(to), "l"(p), "r"(wanted ? 16 : 0), "l"(policy) : "memory");
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void fetch_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <bool kF16>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (kF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// lane (g, t) has elements (g, 2t), (g, 2t + 1) of an 8 x 8 matrix, and gets (2t, g), (2t + 1, g)
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Two e4m3 codes, the lower (upper) half of w, as f16: exact.
__device__ __forceinline__ uint32_t widen_lo(uint32_t w) {
  uint32_t r;
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t w) {
  uint32_t r;
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// What a stretch of chunks is of: a sequence and a tile of the heads that share one of its kv heads.
struct Item {
  int s, kv, h0, rows;  // first of the query heads, how many
  int len, n;           // keys, chunks
};

template <int D, int kType, int HT>
struct TokenShared {
  static constexpr int NW = TokenPlan<D, kType, HT>::kWarps;
  float part_m[2 * NW][HT], part_l[2 * NW][HT];
  Item part_item[2 * NW + 1];  // whose (n = 0: no part); the last: the block's one item, where the host cuts
  int part_first[2 * NW];  // its first chunk
  int last_arrival[2];
  int x0, x1, each, more;     // the block's share; how the blocks' shares are cut
  int item_blocks, in_item;
  int warp_chunks[NW], run_first[NW * 32];  // of more than 32 sequences: chunks of a warp's runs, in front of a thread's run
};
// Parts of the block's warps, two of each: of an item that begins before the warp's stretch (in shared memory of its own), and of one that
// goes on behind it (in the warp's queue, which is empty by then).
template <int D, int kType, int HT>
__device__ __forceinline__ float* part_of(uint8_t* dynamic, int i) {
  using P = TokenPlan<D, kType, HT>;
  return reinterpret_cast<float*>(i & 1 ? dynamic + (i >> 1) * 8192 : dynamic + P::kQueue + (i >> 1) * P::kPart * 4);
}

__device__ __forceinline__ int length_of(const TokenParams& p, int s) { return p.lens ? min(max(p.lens[s], 0), p.cache.cap) : p.cache.cap; }

// The item behind another one.
template <int KC, int HT>
__device__ __forceinline__ Item item_after(const TokenParams& p, Item i) {
  constexpr unsigned full = 0xffffffffu;
  i.h0 += i.rows;
  const int in_group = i.h0 - i.kv * p.group;  // heads of the kv head that are behind us
  if (in_group == p.group && ++i.kv == p.Hkv) {
    const int lane = threadIdx.x & 31;
    i.kv = i.h0 = 0;
    // the next sequence that has keys, 32 at a time; behind the last one: never fetched
    int s0 = i.s + 1;
    i.s = p.S;
    i.len = 0;
    i.n = 0x7fffffff;
#pragma unroll 1
    for (; s0 < p.S; s0 += 32) {
      const int len = s0 + lane < p.S ? length_of(p, s0 + lane) : 0;
      const unsigned some = __ballot_sync(full, len > 0);
      if (some) {
        const int l = __ffs(some) - 1;
        i.s = s0 + l;
        i.len = __shfl_sync(full, len, l);
        i.n = (int)(((unsigned)i.len + KC - 1) / KC);
        break;
      }
    }
  }
  i.rows = min(HT, (i.kv + 1) * p.group - i.h0);
  return i;
}

// Row `row` of the block's parts in `of`, by one warp: offset, sum and 4 dimensions per lane.
template <int D, int kType, int HT>
__device__ __forceinline__ void parts_together(TokenShared<D, kType, HT>& sh, uint8_t* dynamic, unsigned of, int row, float& top, float& sum, float4& o) {
  constexpr unsigned full = 0xffffffffu;
  const int lane = threadIdx.x & 31;
  const bool in = (of >> lane) & 1;
  const float mine = in ? sh.part_m[lane][row] : -CUDART_INF_F;
  top = mine;
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(full, top, off));
  const float weight = in ? exp2_approx(mine - top) : 0.f;
  sum = in ? sh.part_l[lane][row] * weight : 0.f;
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor_sync(full, sum, off);
  o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  while (of) {  // four at a time
    float4 v[4];
    float f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = of ? __ffs(of) - 1 : 0;
      f[k] = __shfl_sync(full, weight, i);
      if (!of) f[k] = 0.f;
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (of) v[k] = *reinterpret_cast<const float4*>(part_of<D, kType, HT>(dynamic, i) + row * D + 4 * (D == 128 ? lane : lane & 15));
      of &= of - 1;  // 0 stays 0
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      o.x = fmaf(v[k].x, f[k], o.x); o.y = fmaf(v[k].y, f[k], o.y); o.z = fmaf(v[k].z, f[k], o.z); o.w = fmaf(v[k].w, f[k], o.w);
    }
  }
}
// A row's result.
template <int D, int kType>
__device__ __forceinline__ void write_row_of(const TokenParams& p, const Item& item, int row, float top, float sum, const float4& o) {
  constexpr bool kF32 = kType == kTypeF32, kF16 = kType == kTypeE4m3;
  const int lane = threadIdx.x & 31;
  const float v_scale = kF16 && p.cache.v_scale ? p.cache.v_scale[item.kv] : 1.f, f = kF32 ? v_scale / sum : __fdividef(v_scale, sum);
  const int head = item.h0 + row;
  const int64_t to = item.s * p.o_b + (int64_t)head * p.o_h + 4 * lane;
  if (D == 128 || lane < 16) {
    if constexpr (kF32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + to) = make_uint2(bf16_pair(o.x * f, o.y * f), bf16_pair(o.z * f, o.w * f));
  }
  if (p.lse && lane == 0) p.lse[(int64_t)item.s * p.Hq + head] = (top + log2f(sum)) * kLn2;
}

__device__ __forceinline__ uint32_t at_rank(const void* p, int rank) {  // the same place in another block of the cluster
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ float peer_float(const float* p, int rank) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at_rank(p, rank)) : "memory");
  return x;
}
__device__ __forceinline__ float4 peer_float4(const float* p, int rank) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at_rank(p, rank)) : "memory");
  return x;
}
// What follows the loop where an item has 2^shift blocks of its own, a cluster: the warps' parts meet in the block's shared memory, the
// blocks' are read from one another's.  (1 sequence of 768 rows, 32 heads, 4 blocks each: 6.5 us; cut by the device and joined through the
// workspace 8.8.)
template <int D, int kType, int HT>
__device__ __noinline__ void join_cluster(const TokenParams& p, uint8_t* dynamic, TokenShared<D, kType, HT>& sh) {
  using P = TokenPlan<D, kType, HT>;
  constexpr int NW = P::kWarps;
  constexpr unsigned full = 0xffffffffu;
  const int warp = __shfl_sync(full, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, blocks = 1 << p.shift;
  float* const slot = reinterpret_cast<float*>(dynamic + P::kBytes);
  __syncthreads();
  const unsigned of = __ballot_sync(full, lane < 2 * NW && sh.part_item[lane].n > 0);  // all of the one item
  const Item it = sh.part_item[2 * NW];
#pragma unroll 1
  for (int row = warp; row < it.rows; row += NW) {
    float top = -CUDART_INF_F, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (of) {
      parts_together<D, kType, HT>(sh, dynamic, of, row, top, sum, o);
      if (blocks == 1) write_row_of<D, kType>(p, it, row, top, sum, o);
    }
    if (D == 128 || lane < 16) *reinterpret_cast<float4*>(slot + row * D + 4 * lane) = o;
    if (lane == 0) { slot[HT * D + row] = top; slot[HT * D + HT + row] = sum; }
  }
  if (blocks == 1) return;
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
  const int rank = (int)blockIdx.x & (blocks - 1);
#pragma unroll 1
  for (int row = rank + (warp << p.shift); row < it.rows; row += NW << p.shift) {
    const bool in = lane < blocks;
    const float mine = in ? peer_float(slot + HT * D + row, lane) : -CUDART_INF_F, sum_mine = in ? peer_float(slot + HT * D + HT + row, lane) : 0.f;
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < blocks) v[i] = peer_float4(slot + row * D + 4 * (D == 128 ? lane : lane & 15), i);
    }
    float top = mine;
#pragma unroll
    for (int off = 4; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(full, top, off));
    top = __shfl_sync(full, top, 0);
    if (top == -CUDART_INF_F) continue;  // no block had a part: no keys, or one chunk, which its warp has written
    const float weight = in ? exp2_approx(mine - top) : 0.f;
    float sum = sum_mine * weight;
#pragma unroll
    for (int off = 4; off >= 1; off >>= 1) sum += __shfl_xor_sync(full, sum, off);
    sum = __shfl_sync(full, sum, 0);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = __shfl_sync(full, weight, i);
      o.x = fmaf(v[i].x, f, o.x); o.y = fmaf(v[i].y, f, o.y); o.z = fmaf(v[i].z, f, o.z); o.w = fmaf(v[i].w, f, o.w);
    }
    write_row_of<D, kType>(p, it, row, top, sum, o);
  }
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");  // no block leaves before its parts are read
}

// What follows the loop over the chunks, a function of its own so that it takes no registers from that loop.
template <int D, int kType, int HT>
__device__ __noinline__ void join_parts(const TokenParams& p, uint8_t* dynamic, TokenShared<D, kType, HT>& sh) {
  using P = TokenPlan<D, kType, HT>;
  constexpr int NW = P::kWarps;
  constexpr unsigned full = 0xffffffffu;
  // the shuffle tells the compiler that the warp branches together, a third of this function's code
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  __syncthreads();  // the share that thread 0 has written, the warps' parts: a warp without chunks has come here at once
  const int x0 = sh.x0, x1 = sh.x1, each = sh.each, more = sh.more;
  auto& part_m = sh.part_m;
  auto& part_l = sh.part_l;
  auto& part_item = sh.part_item;
  auto& part_first = sh.part_first;
  auto& last_arrival = sh.last_arrival;
  auto part_of = [&](int i) { return tsd::part_of<D, kType, HT>(dynamic, i); };
  auto block_of = [&](int x) {
    const bool longer = x < more * (each + 1);
    return (longer ? 0 : more) + (int)((unsigned)(longer ? x : x - more * (each + 1)) / (unsigned)(each + (longer ? 1 : 0)));
  };
  auto blocks_of = [&](int first, int n, int& b_first, int& count) {  // that an item's chunks went to
    b_first = sh.item_blocks ? (int)blockIdx.x - sh.in_item : block_of(first);
    count = sh.item_blocks ? sh.item_blocks : block_of(first + n - 1) - b_first + 1;
  };
  // ---- the block's parts: put together where they are of one sequence, then written out, or, where other blocks have the rest, to the workspace
  auto together = [&](unsigned of, int row, float& top, float& sum, float4& o) { parts_together<D, kType, HT>(sh, dynamic, of, row, top, sum, o); };
  auto write_row = [&](const Item& item, int row, float top, float sum, const float4& o) { write_row_of<D, kType>(p, item, row, top, sum, o); };
  int shared0 = 0, shared1 = 0, n_shared = 0;  // parts with which items of several blocks begin in this one: at most two
  {
    const bool there = lane < 2 * NW && part_item[lane].n > 0;
    const unsigned valid = __ballot_sync(full, there);
    const int id = there ? part_first[lane] : -1;  // items are told apart by their first chunk
    const unsigned below = valid & ((1u << lane) - 1u);
    const int id_before = __shfl_sync(full, id, below ? 31 - __clz(below) : lane);
    const unsigned starts = __ballot_sync(full, there && (!below || id_before != id));
    int turn = 0;  // rows are dealt to the warps in turn
#pragma unroll 1
    for (unsigned st = starts; st; st &= st - 1) {
      const int i = __ffs(st) - 1;
      const unsigned rest = st & (st - 1), of = valid & ~((1u << i) - 1u) & (rest ? (rest & -rest) - 1u : 0xffffffffu);
      const Item it = part_item[i];
      const int first = part_first[i], rows = it.rows;
      const bool whole = first >= x0 && first + it.n <= x1;
      float* slot = p.parts + (2 * (int)blockIdx.x + (first < x0 ? 0 : 1)) * P::kSlot;
#pragma unroll 1
      for (int row = warp >= turn ? warp - turn : warp - turn + NW; row < rows; row += NW) {
        float top, sum;
        float4 o;
        together(of, row, top, sum, o);
        if (whole) {
          write_row(it, row, top, sum, o);
        } else {
          if (D == 128 || lane < 16) *reinterpret_cast<float4*>(slot + row * D + 4 * lane) = o;
          if (lane == 0) { slot[HT * D + row] = top; slot[HT * D + HT + row] = sum; }
        }
      }
      turn = (turn + rows) % NW;
      if (!whole) {
        if (n_shared == 0) shared0 = i;
        else shared1 = i;
        ++n_shared;
      }
    }
  }
  // An item of several blocks: the last of them to arrive puts its parts together.  The barrier puts the block's writes before
  // the arrivals, whose release and acquire take them to the block that arrives last.
  if (n_shared > 0) {
    __syncthreads();
    if (warp < n_shared && lane == 0) {
      const int i0 = warp == 0 ? shared0 : shared1;
      int b_first, n_parts;
      blocks_of(part_first[i0], part_item[i0].n, b_first, n_parts);
      unsigned before;
      asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(p.tickets + b_first) : "memory");
      const bool last = before + 1 == (unsigned)n_parts;
      last_arrival[warp] = last;
      if (last) p.tickets[b_first] = 0;
    }
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < n_shared; ++k) {
      if (!last_arrival[k]) continue;
      const int i0 = k == 0 ? shared0 : shared1;
      const Item it = part_item[i0];
      const int rows = it.rows;
      int b_first, n_parts;
      blocks_of(part_first[i0], it.n, b_first, n_parts);
      // A row by one warp; many parts, and warps to spare: by `subs` warps, each with parts sub, sub + subs, ... , and what they come
      // to meets in the shared memory of their second parts.  32 parts at a time, a lane for the offset and sum of each.
      const int subs = n_parts <= 32 ? 1 : max(1, (int)((unsigned)NW / (unsigned)rows));
      const float* const parts = p.parts + 2 * b_first * P::kSlot;
#pragma unroll 1
      for (int task = warp; task < rows * subs; task += NW) {
        const int sub = (int)((unsigned)task / (unsigned)rows), row = task - sub * rows;
        float top = -CUDART_INF_F, sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        auto part_at = [&](int i) { return parts + max(1, 2 * i) * P::kSlot; };  // the first block's is odd, the others' are even
        const int col = row * D + 4 * (D == 128 ? lane : lane & 15);
#pragma unroll 1
        for (int i0 = sub; i0 < n_parts; i0 += 32 * subs) {
          const int i = i0 + lane * subs;
          const bool in = i < n_parts;
          const float mine = in ? __ldcg(part_at(i) + HT * D + row) : -CUDART_INF_F;
          const float sum_mine = in ? __ldcg(part_at(i) + HT * D + HT + row) : 0.f;
          float weight = 0.f;
#pragma unroll 1
          for (int j = 0; j < 32 && i0 + j * subs < n_parts; j += 8) {
            float4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int k = i0 + (j + u) * subs;
              v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (k < n_parts) v[u] = __ldcg(reinterpret_cast<const float4*>(part_at(k) + col));
            }
            if (j == 0) {
              float to = mine;
#pragma unroll
              for (int off = 16; off >= 1; off >>= 1) to = fmaxf(to, __shfl_xor_sync(full, to, off));
              to = fmaxf(to, top);
              const float alpha = top == to ? 1.f : exp2_approx(top - to);
              weight = in ? exp2_approx(mine - to) : 0.f;
              top = to;
              float all = sum_mine * weight;
#pragma unroll
              for (int off = 16; off >= 1; off >>= 1) all += __shfl_xor_sync(full, all, off);
              sum = fmaf(sum, alpha, all);
              o.x *= alpha; o.y *= alpha; o.z *= alpha; o.w *= alpha;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float f = __shfl_sync(full, weight, j + u);
              o.x = fmaf(v[u].x, f, o.x); o.y = fmaf(v[u].y, f, o.y); o.z = fmaf(v[u].z, f, o.z); o.w = fmaf(v[u].w, f, o.w);
            }
          }
        }
        if (subs == 1) {
          write_row(it, row, top, sum, o);
        } else {
          if (D == 128 || lane < 16) *reinterpret_cast<float4*>(part_of(2 * sub + 1) + col) = o;
          if (lane == 0) { part_m[2 * sub + 1][row] = top; part_l[2 * sub + 1][row] = sum; }
        }
      }
      if (subs == 1) continue;
      __syncthreads();
      const unsigned of = 0xaaaaaaaau & (unsigned)((1ull << (2 * subs)) - 1);
#pragma unroll 1
      for (int row = warp; row < rows; row += NW) {
        float top, sum;
        float4 o;
        together(of, row, top, sum, o);
        write_row(it, row, top, sum, o);
      }
      __syncthreads();
    }
  }
}

// kItems: the host has cut, 2^shift blocks for every item, a cluster of them
template <int D, int kType, int HT, bool kItems>
__global__ void __launch_bounds__(TokenPlan<D, kType, HT>::kWarps * 32, 1) token_attention_kernel(const __grid_constant__ TokenParams p) {
  using P = TokenPlan<D, kType, HT>;
  constexpr int NW = P::kWarps, KC = P::kKeys, NG = P::kGroups, NP = P::kPieces, NT = HT / 8;
  constexpr bool kF32 = kType == kTypeF32, kF16 = kType == kTypeE4m3;  // e4m3 is a subset of f16
  constexpr int kTiles = D / 16;                       // of 16 dimensions
  constexpr bool kSplitRuns = kType == kTypeBf16 && D == 128;  // where the tiles' second dimensions lie
  constexpr int kAcc = kF32 ? HT : kTiles * NT;        // rows of 4 dimensions (fp32), or tiles of 16 dimensions x 8 heads
  extern __shared__ __align__(128) uint8_t dynamic[];  // the queues on whole lines: 16 or 64 bytes beside them cost 4-9 %
  __shared__ TokenShared<D, kType, HT> shared;
  __shared__ __align__(16) float weights[kF32 ? NW : 1][kF32 ? KC : 1][HT];
  static_assert(2 * NW <= 32, "a lane per part");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  constexpr unsigned full = 0xffffffffu;
  TokenParams a = p;
  grid_wait(a.cache.k, a.cache.v, a.cache.table, a.q, a.lens, a.cache.k_scale, a.cache.v_scale);
  const int HI = a.Hkv * a.tiles;  // items of a sequence
  auto length = [&](int s) { return length_of(a, s); };
  auto chunks = [&](int len) { return (int)(((unsigned)len + KC - 1) / KC); };

  int x0, x1, total = 0, run = 0, len0 = 0;  // this block's share [x0, x1) of the chunks, of an item or of all
  Item next;       // the item whose chunk is fetched next, unless the one at hand goes on,
  int next_c = 0;  // and that chunk
  if constexpr (kItems) {
    const int item = (int)(blockIdx.x >> a.shift), in_item = (int)blockIdx.x & ((1 << a.shift) - 1);
    next.s = (int)((unsigned)item / (unsigned)HI);
    const int hi = item - next.s * HI;
    next.kv = a.tiles == 1 ? hi : (int)((unsigned)hi / (unsigned)a.tiles);
    const int tile = hi - next.kv * a.tiles;
    next.h0 = next.kv * a.group + tile * HT;
    next.rows = min(HT, a.group - tile * HT);
    next.len = length(next.s);
    next.n = chunks(next.len);
    const int even = next.n >> a.shift, rest = next.n & ((1 << a.shift) - 1);
    x0 = in_item * even + min(in_item, rest);
    x1 = x0 + even + (in_item < rest ? 1 : 0);
    if (tid == 0) shared.part_item[2 * NW] = next;
  } else {
    // ---- this block's share [x0, x1) of all chunks (fewer than 2^30: checked on the host)
    // Up to 32 sequences: a lane each, every warp for itself.  More: a thread for a run of them, whose chunks are added up over the block.
    len0 = lane < a.S ? length(lane) : 0;  // of the first 32 sequences
    run = a.S <= 32 ? 0 : (int)((unsigned)(a.S + NW * 32 - 1) / (NW * 32));
    if (run == 0) {
      total = __reduce_add_sync(full, chunks(len0));
    } else {
      int mine = 0;
#pragma unroll 4
      for (int k = 0; k < run; ++k) mine += tid * run + k < a.S ? chunks(length(tid * run + k)) : 0;
      int upto = mine;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(full, upto, off);
        if (lane >= off) upto += o;
      }
      if (lane == 31) shared.warp_chunks[warp] = upto;
      __syncthreads();
      const int of_warp = lane < NW ? shared.warp_chunks[lane] : 0;
      total = __reduce_add_sync(full, of_warp);
      shared.run_first[tid] = upto - mine + __reduce_add_sync(full, lane < warp ? of_warp : 0);
      __syncthreads();
    }
    total *= HI;
    // The chunks of up to 32 sequences are cut item by item, into equal pieces, one per block: then a block has parts of one item only and one
    // arrival to wait for, and fewer blocks than SMs have the memory's rate too.  That is worth pieces a quarter longer than an
    // even share.  Where there is little to do a piece is a chunk for each of the block's warps, and two if that leaves no item to
    // more than one block.  Otherwise, and for more sequences, the blocks take `each` chunks, the first `more` of them one more, wherever
    // that cuts the items.  (16 sequences of 2048, 8 kv heads, in 128 blocks instead of 148: 27.4 us instead of 30.8; 120 heads of one sequence
    // of 8192 in 120: 78.2, 82.5; with pieces a half longer 50 heads in 100 blocks 73.6, 72.1, in e4m3 50.4, 44.0.  8 items of 16 chunks, in
    // 8 blocks instead of 11: 7.5 us instead of 10.2; 32 items of 8 chunks, in 32 blocks instead of 22: 6.5 instead of 11.1.  A third chunk
    // per warp is not worth it: 36 chunks 9.5 us in one block, 8.9 in three.)
    const int n0 = chunks(len0), longest = __reduce_max_sync(full, n0);
    const int for_warps = a.S <= 32 ? HI * __reduce_add_sync(full, (n0 + NW - 1) / NW) : (total + NW - 1) / NW;
    const int most_blocks = max(1, min((int)gridDim.x, for_warps));
    const int each = (int)((unsigned)total / (unsigned)most_blocks), more = total - each * most_blocks;
    int item_blocks = 0, in_item = 0;  // of the block's item, if they are cut one by one: blocks, and which of them this is
    int pieces = 0;                         // of each item of the lane's sequence
    if (a.S <= 32 && total > 0) {
      // A quotient that is off by a rounding is as good, as long as no piece is empty: a block without chunks would never arrive.
      auto fit = [&](int piece) {
        pieces = min(n0, max(1, (int)ceilf(__fdividef((float)n0, (float)piece))));
        return HI * __reduce_add_sync(full, pieces) <= most_blocks;
      };
      int lo = each + (more > 0) - 1, hi = each + 2 + each / kAlignSlack;  // the smallest that fits is looked for in (lo, hi]
      if (for_warps == most_blocks) { hi = NW; lo = hi - 1; }
      if (longest <= 2 * NW && HI * __popc(__ballot_sync(full, n0 > 0)) <= most_blocks) { hi = longest; lo = hi - 1; }
      if (fit(hi)) {
        item_blocks = 1;
        int best = pieces;
#pragma unroll 1
        for (int tries = 0; tries < 5 && lo + 1 < hi; ++tries) {
          const int mid = (lo + hi) >> 1;
          if (fit(mid)) { hi = mid; best = pieces; }
          else lo = mid;
        }
        pieces = best;
      }
    }
    if (item_blocks) {
      int blocks_upto = pieces * HI, chunks_upto = n0 * HI;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(full, blocks_upto, off), c = __shfl_up_sync(full, chunks_upto, off);
        if (lane >= off) { blocks_upto += o; chunks_upto += c; }
      }
      const unsigned hit = __ballot_sync(full, blocks_upto > (int)blockIdx.x);
      const int l = hit ? __ffs(hit) - 1 : 0;
      item_blocks = __shfl_sync(full, pieces, l);
      const int n = __shfl_sync(full, n0, l), b = (int)blockIdx.x - (__shfl_sync(full, blocks_upto, l) - item_blocks * HI);
      const int hi = hit ? (int)((unsigned)b / (unsigned)item_blocks) : 0;
      in_item = b - hi * item_blocks;
      const int first = __shfl_sync(full, chunks_upto, l) - n * HI + hi * n;
      const int even = hit ? (int)((unsigned)n / (unsigned)item_blocks) : 0, rest = n - even * item_blocks;
      x0 = hit ? first + in_item * even + min(in_item, rest) : total;
      x1 = hit ? x0 + even + (in_item < rest ? 1 : 0) : total;
    } else {
      const int b = min((int)blockIdx.x, most_blocks);
      x0 = b * each + min(b, more);
      x1 = b == most_blocks ? total : x0 + each + (b < more ? 1 : 0);
    }
    if (tid == 0) {
      shared.x0 = x0; shared.x1 = x1; shared.each = each; shared.more = more;
      shared.item_blocks = item_blocks; shared.in_item = in_item;
    }
  }
  // and its warps an even share of that, [w0, w1) for this one
  const unsigned share = (unsigned)(x1 - x0) / NW, longer = (unsigned)(x1 - x0) % NW;
  const int w0 = x0 + (int)(warp * share + min((unsigned)warp, longer)), w1 = w0 + (int)(share + (warp < (int)longer ? 1 : 0));

  // ---- where chunk w0 lies
  if constexpr (kItems) {
    next_c = w0;
  } else {
    int before = 0;
    next.s = 0;
    next.len = 0;
    if (run == 0) {
      const int mine = chunks(len0) * HI;
      int upto = mine;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(full, upto, off);
        if (lane >= off) upto += o;
      }
      const unsigned hit = __ballot_sync(full, upto > w0);
      if (hit) {
        next.s = __ffs(hit) - 1;
        next.len = __shfl_sync(full, len0, next.s);
        before = __shfl_sync(full, upto - mine, next.s);
      }
    } else if (w0 < total) {
      int lo = 0, hi = NW * 32 - 1;  // the last run that begins at or before w0: no run of empty sequences begins behind it
#pragma unroll 1
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (shared.run_first[mid] * HI <= w0) lo = mid;
        else hi = mid - 1;
      }
      before = shared.run_first[lo] * HI;
      next.s = lo * run;
      next.len = length(next.s);
#pragma unroll 1
      while (before + chunks(next.len) * HI <= w0) {  // ends: the chunk exists
        before += chunks(next.len) * HI;
        next.len = length(++next.s);
      }
    }
    next.n = max(chunks(next.len), 1);
    const int hi = (int)((unsigned)(w0 - before) / (unsigned)next.n);
    next_c = (w0 - before) - hi * next.n;
    next.kv = a.tiles == 1 ? hi : (int)((unsigned)hi / (unsigned)a.tiles);
    const int tile = hi - next.kv * a.tiles;
    next.h0 = next.kv * a.group + tile * HT;
    next.rows = min(HT, a.group - tile * HT);
  }
  const int row_mask = (1 << a.cache.shift) - 1;
  const int64_t row_bytes = a.cache.ps_r * P::kSize, page_bytes = a.cache.ps_p * P::kSize, head_bytes = a.cache.ps_h * P::kSize;
  // lane i < NG: the table's entry for the chunk's keys [8 i, 8 i + 8)
  auto entry_of = [&](const Item& i, int c) {
    const int key = c * KC + 8 * lane;
    return lane < NG && key < i.len ? a.cache.table[i.s * a.cache.table_stride + (key >> a.cache.shift)] : -1;
  };
  bool bad_page = false;
  // The warp's queue: 4 KB of K, 4 KB of V.  They are fetched along the rows (an instruction that touches whole 128-byte lines: in the order
  // in which the lanes want V, 32 bytes of a line at a time, the same loop without any arithmetic reads 5.0 TB/s instead of
  // 6.9) and read back in the products' order, 16-byte pieces of a 128-byte line exchanged by row so that both orders of reading are free
  // of bank conflicts (8 lanes read 4 pieces of 2 rows of K, 2 pieces of 4 rows of V).
  constexpr int kLine = P::kRow / 16, kRowsAtOnce = 32 / kLine;  // pieces per row, rows per instruction
  constexpr auto swizzle = [](int row) {                         // what a row's pieces are exchanged by: linear in the row's bits
    return P::kRow == 64 ? (row >> 1) & 3 : ((row ^ (row >> 1)) & 1) << 2 | ((row >> 2) & 1) << 1;
  };
  uint8_t* const queue = dynamic + warp * 8192;
  const int my_row = lane / kLine, my_piece = lane % kLine;
  const uint32_t lane_to = my_row * P::kRow + (my_piece ^ swizzle(my_row)) * 16;
  const uint32_t queue_at = (uint32_t)__cvta_generic_to_shared(queue);
  const int64_t lane_from = my_row * row_bytes + 16 * my_piece;
  // `at`: lane i < NG, where the chunk's 8 keys from 8 i on begin (from k or v on), -1 where there is no page; `left`: how many keys count
  // Much data is read past what else L2 holds, the code of what follows the loop above all: 0.8-2 us per call.  Data that may still be there
  // from the call before is left to it (12.6 MB, read again and again: 8.8 us, read past it 9.6).
  uint64_t policy;
  if (total >= kReadPast) asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  else asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
  auto fetch = [&](int64_t at, int left, const void* pages, uint32_t to) {
#pragma unroll
    for (int nb = 0; nb < NG; ++nb) {
      const int64_t from = __shfl_sync(full, at, nb);
      const uint8_t* p = static_cast<const uint8_t*>(pages) + (from < 0 ? 0 : from) + lane_from;
      const int here = from < 0 ? 0 : left - 8 * nb - my_row;  // how many of the group's keys, from this lane's first one on
#pragma unroll
      for (int j = 0; j < 8 / kRowsAtOnce; ++j) {
        const int row0 = 8 * nb + j * kRowsAtOnce;
        fetch16(to + (lane_to ^ (swizzle(row0) * 16)) + row0 * P::kRow, p, j * kRowsAtOnce < here, policy);
        p += kRowsAtOnce * row_bytes;
      }
    }
  };
  // K: 16 bytes at 64 pc + 16 t of key 8 nb + g.  V: of the lane's keys 16 mt + 2t + {0, 1, 8, 9}, number i, 16 bytes at 128 h + 16 g (rows of 64
  // bytes: the 16 that hold its 8)
  const uint8_t* const k_lane = queue + g * P::kRow;
  const int k_to = (t ^ swizzle(g)) * 16;
  const uint8_t* const v_lane = queue + 4096 + 2 * t * P::kRow;
  const int v_to = ((P::kRow == 64 ? g >> 1 : g) ^ swizzle(2 * t)) * 16;
  auto k_piece = [&](int nb, int pc) { return *reinterpret_cast<const uint4*>(k_lane + 8 * nb * P::kRow + (k_to ^ ((pc & 1) * 64)) + (pc >> 1) * 128); };
  auto v_piece = [&](int mt, int i, int h) {
    return *reinterpret_cast<const uint4*>(v_lane + (16 * mt + (i & 1) + 8 * (i >> 1)) * P::kRow + (v_to ^ (swizzle(i & 1) * 16)) + h * 128);
  };

  // the lane's part of the query rows of a (sequence, head tile): of head g (and g + 8), laid out as the keys are; fp32 reads them where they are
  uint32_t qr[kF32 ? 1 : NT][kF32 ? 1 : D / 8];
  float score_scale[kF16 ? 2 * NT : 1];  // e4m3: of the heads whose scores the lane gets
  auto load_q = [&](const Item& i) {
    if constexpr (!kF32) {
      constexpr int E = 16 / P::kSize;  // elements of a lane's piece
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = g + 8 * nt;
        const __nv_bfloat16* row = static_cast<const __nv_bfloat16*>(a.q) + i.s * a.q_b + (int64_t)(i.h0 + r) * a.q_h;
#pragma unroll
        for (int pc = 0; pc < NP; ++pc)
#pragma unroll
          for (int e = 0; e < E / 8; ++e) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < i.rows) v = *reinterpret_cast<const uint4*>(row + pc * 4 * E + t * E + e * 8);
#pragma unroll
            for (int k = 0; k < 4; ++k) qr[nt][(pc * (E / 8) + e) * 4 + k] = word(v, k);
          }
      }
    }
  };
  auto take_q = [&](const Item& item) {
    const float scale = a.scale_log2e * (kF16 && a.cache.k_scale ? a.cache.k_scale[item.kv] : 1.f);
    if constexpr (!kF16) {
      score_scale[0] = scale;
    } else {
      // bf16 -> f16, the row scaled by a power of 2 that puts its largest element at 2^13: exact for elements down to 2^-27 of
      // that one, and off by 2^-38 of it below
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(qr[nt][i] << 16)), fabsf(__uint_as_float(qr[nt][i] & 0xffff0000u))));
        top = fmaxf(top, __shfl_xor_sync(full, top, 1));
        top = fmaxf(top, __shfl_xor_sync(full, top, 2));
        const int up = min(max(267 - (int)(__float_as_uint(top) >> 23), 1), 240);  // exponent field of that power
        const float f = __uint_as_float((uint32_t)up << 23), back = __uint_as_float((uint32_t)(254 - up) << 23);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) qr[nt][i] = f16_pair(__uint_as_float(qr[nt][i] << 16) * f, __uint_as_float(qr[nt][i] & 0xffff0000u) * f);
#pragma unroll
        for (int i = 0; i < 2; ++i) score_scale[2 * nt + i] = scale * __shfl_sync(full, back, (2 * t + i) * 4);
      }
    }
  };

  float acc[kAcc][4];
  // heads 8 nt + 2t, + 1: the exponent offset, the same in all lanes that share the heads, and the sum of the lane's own keys' weights;
  // fp32: of row lane % HT, both equal in the lanes that share it
  float m[kF32 ? 1 : 2 * NT], l[kF32 ? 1 : 2 * NT];

  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < kAcc; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(m) / 4); ++i) { m[i] = kLowest; l[i] = 0.f; }
  };
  // What an item's chunks have come to so far: put aside as part i of the block, or, if they are all of it, written out.
  auto put_aside = [&](const Item& item, int first, int i) {
    float* o = part_of<D, kType, HT>(dynamic, i);
    const int rows = item.rows;
    if (lane == 0) { shared.part_item[i] = item; shared.part_first[i] = first; }
    if constexpr (kF32) {
#pragma unroll
      for (int r = 0; r < HT; ++r)
        if (r < rows && (D == 128 || lane < 16)) *reinterpret_cast<float4*>(o + r * D + 4 * lane) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
      if (lane < HT) { shared.part_m[i][lane] = m[0]; shared.part_l[i][lane] = l[0]; }
    } else {
#pragma unroll
      for (int h = 0; h < 2 * NT; ++h) {
        const int head = 8 * (h >> 1) + 2 * t + (h & 1);
        if (g == 0) { shared.part_m[i][head] = m[h]; shared.part_l[i][head] = l[h]; }
        if (head < rows) {
#pragma unroll
          for (int run = 0; run < 2; ++run)
#pragma unroll
            for (int j = 0; j < kTiles; j += 4) {
              float v[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) v[k] = acc[(h >> 1) * kTiles + j + k][2 * run + (h & 1)];
              *reinterpret_cast<float4*>(o + head * D + (kSplitRuns ? 64 * run + 8 * g : (2 * g + run) * kTiles) + j) = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
      }
    }
  };
  auto write_out = [&](const Item& item) {
    const int rows = item.rows;
    const float v_scale = kF16 && a.cache.v_scale ? a.cache.v_scale[item.kv] : 1.f;
    const int64_t to = item.s * a.o_b + (int64_t)item.h0 * a.o_h, lse_to = (int64_t)item.s * a.Hq + item.h0;
    if constexpr (kF32) {
#pragma unroll
      for (int r = 0; r < HT; ++r) {
        const float f = 1.f / __shfl_sync(full, l[0], r);
        if (r < rows && (D == 128 || lane < 16))
          *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to + r * a.o_h + 4 * lane) = make_float4(acc[r][0] * f, acc[r][1] * f, acc[r][2] * f, acc[r][3] * f);
      }
      if (a.lse && lane < rows) a.lse[lse_to + lane] = (m[0] + log2f(l[0])) * kLn2;
    } else {
#pragma unroll
      for (int h = 0; h < 2 * NT; ++h) {
        const int head = 8 * (h >> 1) + 2 * t + (h & 1);
        if (head < rows) {
          const float f = __fdividef(v_scale, l[h]);  // 2 ulp
          __nv_bfloat16* row = static_cast<__nv_bfloat16*>(a.out) + to + head * a.o_h;
#pragma unroll
          for (int run = 0; run < 2; ++run) {
            uint32_t w[kTiles / 2];
#pragma unroll
            for (int j = 0; j < kTiles / 2; ++j)
              w[j] = bf16_pair(acc[(h >> 1) * kTiles + 2 * j][2 * run + (h & 1)] * f, acc[(h >> 1) * kTiles + 2 * j + 1][2 * run + (h & 1)] * f);
            __nv_bfloat16* at = row + (kSplitRuns ? 64 * run + 8 * g : (2 * g + run) * kTiles);
            if constexpr (kTiles == 8) *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
          }
          if (a.lse && g == 0) a.lse[lse_to + head] = (m[h] + __log2f(l[h])) * kLn2;
        }
      }
    }
  };

  // ---- the warp's chunks.  The round before the first one only fetches.
  if (lane < 2) shared.part_item[2 * warp + lane].n = 0;
  __syncwarp();
  Item item = next;                                     // at hand, and its chunk;
  int c = 0, left = 0;                                  // how many of the chunk's keys count
  int entry = -1;                                       // the table's entries for the chunk behind it,
  int next_entry = w0 < w1 ? entry_of(next, next_c) : -1;  // and for the next item's
  bool fresh = false;                                   // the item's queries have just been asked for
  int x = w0 - 1;
  asm volatile("" : "+r"(x));  // the compiler is not to lay the loop out twice for that round
#pragma unroll 1
  for (; x < w1; ++x) {
    const bool real = x >= w0, more_chunks = x + 1 < w1, ends = !real || c + 1 == item.n;  // of the warp; the item
    const int rows = item.rows;
    int64_t at = -1;
    int then = 0, then_left = 0;  // the chunk that is fetched in this round
    auto fetch_next_k = [&] {
      if (more_chunks) {
        then = ends ? next_c : c + 1;
        const int kv = ends ? next.kv : item.kv, e = ends ? next_entry : entry, key = then * KC + 8 * lane;
        then_left = (ends ? next.len : item.len) - then * KC;
        const bool there = e >= 0 && e < a.cache.n_pages;
        bad_page |= lane < NG && 8 * lane < then_left && !there;
        at = there ? (int64_t)e * page_bytes + (int64_t)(key & row_mask) * row_bytes + (int64_t)kv * head_bytes : -1;
        fetch(at, then_left, a.cache.k, queue_at);
        if (ends) load_q(next);
      }
      fetch_commit();
    };
    auto fetch_next_v = [&] {
      if (more_chunks) {
        fetch(at, then_left, a.cache.v, queue_at + 4096);
        if (ends) entry = entry_of(next, then + 1);
        else entry = entry_of(item, then + 1);
      }
      fetch_commit();
    };
    // While a chunk is worked on, two groups of fetches are under way: its K and its V, then its V and the next one's K.
    float sc[kF32 ? 1 : NG / 2][NT][4];  // scores of keys 16 mt + g and + 8, heads 8 nt + 2t and + 1; then the weights
    if (real) {
      fetch_wait<1>();
      __syncwarp();
      if (fresh) {
        clear();
        take_q(item);
      }
      if constexpr (!kF32) {
        // ---------------------------------------------------------------- scores
#pragma unroll
        for (int mt = 0; mt < NG / 2; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) sc[mt][nt][0] = sc[mt][nt][1] = sc[mt][nt][2] = sc[mt][nt][3] = 0.f;
#pragma unroll
        for (int pc = 0; pc < NP; ++pc) {
#pragma unroll
          for (int mt = 0; mt < NG / 2; ++mt) {
            const uint4 k0 = k_piece(2 * mt, pc), k8 = k_piece(2 * mt + 1, pc);
            if constexpr (kType == kTypeBf16) {
#pragma unroll
              for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                  mma<kF16>(sc[mt][nt], word(k0, 2 * e), word(k8, 2 * e), word(k0, 2 * e + 1), word(k8, 2 * e + 1), qr[nt][pc * 4 + 2 * e], qr[nt][pc * 4 + 2 * e + 1]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t a0 = widen_lo(word(k0, e)), a1 = widen_lo(word(k8, e)), a2 = widen_hi(word(k0, e)), a3 = widen_hi(word(k8, e));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<kF16>(sc[mt][nt], a0, a1, a2, a3, qr[nt][pc * 8 + 2 * e], qr[nt][pc * 8 + 2 * e + 1]);
              }
            }
          }
        }
      } else {
        // ---------------------------------------------------------------- fp32 scores: 4 lanes per key
        const float* q32 = static_cast<const float*>(a.q) + item.s * a.q_b + (int64_t)item.h0 * a.q_h;
        uint4 kr[NG][NP];
#pragma unroll
        for (int nb = 0; nb < NG; ++nb)
#pragma unroll
          for (int pc = 0; pc < NP; ++pc) kr[nb][pc] = k_piece(nb, pc);
#pragma unroll 1
        for (int r = 0; r < rows; ++r) {
          float z[NG];
#pragma unroll
          for (int nb = 0; nb < NG; ++nb) z[nb] = 0.f;
#pragma unroll
          for (int pc = 0; pc < NP; ++pc) {
            const float4 qv = __ldg(reinterpret_cast<const float4*>(q32 + r * a.q_h + 16 * pc + 4 * t));
#pragma unroll
            for (int nb = 0; nb < NG; ++nb) {
              z[nb] = fmaf(qv.x, __uint_as_float(kr[nb][pc].x), z[nb]);
              z[nb] = fmaf(qv.y, __uint_as_float(kr[nb][pc].y), z[nb]);
              z[nb] = fmaf(qv.z, __uint_as_float(kr[nb][pc].z), z[nb]);
              z[nb] = fmaf(qv.w, __uint_as_float(kr[nb][pc].w), z[nb]);
            }
          }
#pragma unroll
          for (int nb = 0; nb < NG; ++nb) {
            z[nb] += __shfl_xor_sync(full, z[nb], 1);
            z[nb] += __shfl_xor_sync(full, z[nb], 2);
            if (t == 0) weights[warp][8 * nb + g][r] = 8 * nb + g < left ? z[nb] * score_scale[0] : -CUDART_INF_F;
          }
        }
      }
      __syncwarp();
    }
    fetch_next_k();  // in the place of the K that has been used
    if (real) {
      fetch_wait<1>();
      __syncwarp();
      if constexpr (!kF32) {
        // ---------------------------------------------------------------- weights
        bool passed = false;
#pragma unroll
        for (int mt = 0; mt < NG / 2; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[mt][nt][e] *= score_scale[kF16 ? 2 * nt + (e & 1) : 0];
        if (left < KC) {
#pragma unroll
          for (int mt = 0; mt < NG / 2; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (16 * mt + 8 * (e >> 1) + g >= left) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) sc[mt][nt][e] = -CUDART_INF_F;
              }
        }
        float top[2 * NT];
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
          top[i] = -CUDART_INF_F;
#pragma unroll
          for (int mt = 0; mt < NG / 2; ++mt) top[i] = fmaxf(top[i], fmaxf(sc[mt][i >> 1][i & 1], sc[mt][i >> 1][2 + (i & 1)]));
          passed |= top[i] > m[i] + (kBelow<kType> + kSlack);
        }
        if (__any_sync(full, passed)) {
#pragma unroll
          for (int i = 0; i < 2 * NT; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(full, top[i], 4));
            top[i] = fmaxf(top[i], __shfl_xor_sync(full, top[i], 8));
            top[i] = fmaxf(top[i], __shfl_xor_sync(full, top[i], 16));
            const float to = fmaxf(m[i], top[i] - kBelow<kType>);
            const float alpha = m[i] == to ? 1.f : exp2_approx(m[i] - to);
            m[i] = to;
            l[i] *= alpha;
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
              acc[(i >> 1) * kTiles + j][i & 1] *= alpha;
              acc[(i >> 1) * kTiles + j][2 + (i & 1)] *= alpha;
            }
          }
        }
#pragma unroll
        for (int mt = 0; mt < NG / 2; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float& z = sc[mt][nt][e];
              z = exp2_approx(z - m[2 * nt + (e & 1)]);
              l[2 * nt + (e & 1)] += z;
            }
        // ---------------------------------------------------------------- weighted sum of the values
#pragma unroll
        for (int mt = 0; mt < NG / 2; ++mt) {
          uint32_t b0[NT], b1[NT], r0[NT], r1[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const float(&w)[4] = sc[mt][nt];
            split_pair<kF16>(w[0], w[1], b0[nt], r0[nt]);
            split_pair<kF16>(w[2], w[3], b1[nt], r1[nt]);
            b0[nt] = transposed(b0[nt]);
            b1[nt] = transposed(b1[nt]);
            r0[nt] = transposed(r0[nt]);
            r1[nt] = transposed(r1[nt]);
          }
          auto step = [&](int j, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma<kF16>(acc[nt * kTiles + j], a0, a1, a2, a3, b0[nt], b1[nt]);
              mma<kF16>(acc[nt * kTiles + j], a0, a1, a2, a3, r0[nt], r1[nt]);
            }
          };
          if constexpr (kType == kTypeBf16) {
            constexpr int H2 = D / 64;  // pieces of a key
            uint4 u[4][H2];             // keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int h = 0; h < H2; ++h) u[i][h] = v_piece(mt, i, h);
            auto pair = [&](int i, int h, int j) {  // element j of the piece, of keys i and i + 1
              return __byte_perm(word(u[i][h], j >> 1), word(u[i + 1][h], j >> 1), j & 1 ? 0x7632 : 0x5410);
            };
            // tile j: dimensions 8 g + j and 64 + 8 g + j (64-wide heads: 8 g + j and 8 g + 4 + j)
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
              if constexpr (D == 128) step(j, pair(0, 0, j), pair(0, H2 - 1, j), pair(2, 0, j), pair(2, H2 - 1, j));
              else step(j, pair(0, 0, j), pair(0, 0, j + 4), pair(2, 0, j), pair(2, 0, j + 4));
            }
          } else {
            // a lane's dimensions of a key: 16 bytes, or with 64 dimensions the lower or the upper 8 of them
            uint32_t u[4][D / 32];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint4 v = v_piece(mt, i, 0);
#pragma unroll
              for (int k = 0; k < D / 32; ++k) u[i][k] = D == 64 ? (g & 1 ? word(v, 2 + k) : word(v, k)) : word(v, k);
            }
            auto two = [&](int i, int j) {  // bytes j and j + 1 of keys i and i + 1, key by key
              return __byte_perm(u[i][j >> 2], u[i + 1][j >> 2], j & 2 ? 0x7362 : 0x5140);
            };
            // tile j: dimensions 16 g + j and 16 g + 8 + j (64-wide heads: 8 g + j and 8 g + 4 + j)
#pragma unroll
            for (int j = 0; j < kTiles; j += 2) {
              const uint32_t w0 = two(0, j), w1 = two(0, j + kTiles), w2 = two(2, j), w3 = two(2, j + kTiles);
              step(j, widen_lo(w0), widen_lo(w1), widen_lo(w2), widen_lo(w3));
              step(j + 1, widen_hi(w0), widen_hi(w1), widen_hi(w2), widen_hi(w3));
            }
          }
        }
      } else {
        // row lane % HT, keys lane / HT, + 32 / HT, ...
        {
          constexpr int KL = 32 / HT;  // keys that the lanes take at once
          const int r = lane % HT;
          float z[KC / KL], top = -CUDART_INF_F;
#pragma unroll
          for (int i = 0; i < KC / KL; ++i) {
            z[i] = r < rows ? weights[warp][i * KL + lane / HT][r] : 0.f;
            top = fmaxf(top, z[i]);
          }
          if (__any_sync(full, top > m[0] + kSlack)) {
#pragma unroll
            for (int off = HT; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(full, top, off));
            const float to = fmaxf(m[0], top), alpha = m[0] == to ? 1.f : exp2f(m[0] - to);
            m[0] = to;
            l[0] *= alpha;
#pragma unroll
            for (int i = 0; i < HT; ++i) {
              const float f = __shfl_sync(full, alpha, i);
              acc[i][0] *= f; acc[i][1] *= f; acc[i][2] *= f; acc[i][3] *= f;
            }
          }
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < KC / KL; ++i) {
            z[i] = exp2f(z[i] - m[0]);
            sum += z[i];
            weights[warp][i * KL + lane / HT][r] = z[i];
          }
#pragma unroll
          for (int off = HT; off < 32; off <<= 1) sum += __shfl_xor_sync(full, sum, off);
          l[0] += sum;
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int in = D == 128 ? i : 2 * i + (lane >> 4);
          const uint4 vw = *reinterpret_cast<const uint4*>(queue + 4096 + in * P::kRow + ((D == 128 ? lane : lane & 15) ^ swizzle(in)) * 16);
          const float4 v = make_float4(__uint_as_float(vw.x), __uint_as_float(vw.y), __uint_as_float(vw.z), __uint_as_float(vw.w));
#pragma unroll
          for (int r4 = 0; r4 < HT / 4; ++r4) {
            if (r4 * 4 < rows) {
              const float4 w4 = *reinterpret_cast<const float4*>(&weights[warp][in][4 * r4]);
              const float w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float(&o)[4] = acc[4 * r4 + e];
                o[0] = fmaf(w[e], v.x, o[0]);
                o[1] = fmaf(w[e], v.y, o[1]);
                o[2] = fmaf(w[e], v.z, o[2]);
                o[3] = fmaf(w[e], v.w, o[3]);
              }
            }
          }
        }
      }
      __syncwarp();
    }
    fetch_next_v();
    if (real) {
      if (ends || !more_chunks) {  // the item's last chunk, or the warp's
        if constexpr (kF32) {
          if (D == 64) {  // the two halves of the warp had different keys
#pragma unroll
            for (int r = 0; r < HT; ++r)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[r][i] += __shfl_xor_sync(full, acc[r][i], 16);
          }
        } else {
#pragma unroll
          for (int h = 0; h < 2 * NT; ++h) {
            l[h] += __shfl_xor_sync(full, l[h], 4);
            l[h] += __shfl_xor_sync(full, l[h], 8);
            l[h] += __shfl_xor_sync(full, l[h], 16);
          }
        }
        const int first = x - c;
        if (first < w0) put_aside(item, first, 2 * warp);
        else if (ends) write_out(item);
        else put_aside(item, first, 2 * warp + 1);
      }
    }
    left = then_left;
    c = then;
    fresh = ends;
    if (ends && more_chunks) {
      item = next;
      if (!kItems && x + 1 + item.n - c < w1) {  // the warp has chunks of another one behind it
        next = item_after<KC, HT>(p, next);
        next_c = 0;
        next_entry = entry_of(next, 0);
      }
    }
  }

  if constexpr (kItems) join_cluster<D, kType, HT>(p, dynamic, shared);
  else join_parts<D, kType, HT>(p, dynamic, shared);

  // sequences without keys
#pragma unroll 1
  for (int s = (int)(blockIdx.x + gridDim.x * warp); s < a.S; s += (int)gridDim.x * NW) {
    if (length(s) > 0) continue;
#pragma unroll 1
    for (int h = 0; h < a.Hq; ++h) {
      if (a.lse && lane == 0) a.lse[(int64_t)s * a.Hq + h] = -CUDART_INF_F;
      if (lane < D * (kF32 ? 4 : 2) / 16)
        reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.out) + (s * a.o_b + h * a.o_h) * (kF32 ? 4 : 2))[lane] = make_uint4(0, 0, 0, 0);
    }
  }
  if (__any_sync(full, bad_page) && lane == 0 && a.status) atomicOr(a.status, TSD_STATUS_BAD_INDEX);
}

// Heads per tile, the columns of a product: 8 where they suffice; 16 are two products, their accumulators for 8 warps instead of 12.
static int head_tile(int group) { return group <= 8 ? 8 : 16; }

// The kernel's dynamic shared memory limit, an attribute per device.
template <int D, int kType, int HT, bool kItems>
static cudaError_t allow_smem() {
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static bool done[kMaxDevices];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (done[dev]) return cudaSuccess;
  e = cudaFuncSetAttribute(token_attention_kernel<D, kType, HT, kItems>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           TokenPlan<D, kType, HT>::template kBytesFor<kItems>);
  done[dev] = e == cudaSuccess;
  return e;
}

template <int D, int kType, int HT, bool kItems>
static int launch_token(const TokenParams& p, int64_t grid, cudaStream_t stream) {
  using P = TokenPlan<D, kType, HT>;
  cudaError_t e = allow_smem<D, kType, HT, kItems>();
  if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(token_attention_kernel)");
  e = launch_clusters(1 << p.shift, token_attention_kernel<D, kType, HT, kItems>, dim3((unsigned)grid), dim3(P::kWarps * 32), P::template kBytesFor<kItems>,
                      stream, p);
  return e != cudaSuccess ? cuda_fail(e, "token_attention_kernel") : TSD_OK;
}

template <int D, int kType, int HT>
static int launch_token(TokenParams p, cudaStream_t stream) {
  using P = TokenPlan<D, kType, HT>;
  const int64_t items = (int64_t)p.S * p.Hkv * p.tiles, per_item = (p.cache.cap + P::kKeys - 1) / P::kKeys;
  const int64_t most = items * per_item;  // chunks, if every sequence were full
  if (most >= (1 << 30)) return TSD_ERR_UNSUPPORTED;
  // Short caches: the host cuts, 1, 2, 4 or 8 blocks for every item, a cluster that joins in shared memory and needs to look at one length
  // only.  One block where its warps have a chunk each, otherwise as many as there is room for (clusters of 4 find SMs for 128
  // blocks, clusters of 8 for fewer than 128: 16 of them take 15.3 us where 16 items cut by the device take 11.3), as long as a warp
  // gets no more than three chunks.  Clusters against the device's cut: 32 items of 48 chunks 6.5 us, 8.8; 8 of 16 5.6, 7.5 (in 2 blocks 6.2);
  // 32 of 8, in a block each, 4.9, 6.3 (in 2 blocks 5.7); 8 of 256 9.4, 11.0; 8 of 375 (four chunks) 11.1, 11.4, and 4 of 375
  // 11.3, 11.0.  Where lengths are ragged and three chunks long it can lose: 4 sequences of up to 2000, 4 kv heads, 12.2, 10.8.
  const auto room = [&](int shift) { return items << shift <= (shift == 3 ? 96 : shift == 2 ? 128 : kTokenBlocks); };
  p.shift = 0;
  while (per_item > P::kWarps && p.shift < 3 && room(p.shift + 1)) ++p.shift;
  if (room(p.shift) && per_item <= (int64_t)3 * P::kWarps << p.shift) return launch_token<D, kType, HT, true>(p, items << p.shift, stream);
  p.shift = 0;
  // a chunk for each of a block's warps; up to 32 sequences may be cut item by item
  const int64_t grid = std::min<int64_t>(kTokenBlocks, p.S <= 32 ? items * ((per_item + P::kWarps - 1) / P::kWarps) : (most + P::kWarps - 1) / P::kWarps);
  return launch_token<D, kType, HT, false>(p, std::max<int64_t>(grid, 1), stream);
}

template <int D>
static int launch_token(int type, const TokenParams& p, cudaStream_t stream) {
  const bool wide = head_tile(p.group) == 16;
  if (type == TSD_F32) return wide ? launch_token<D, kTypeF32, 16>(p, stream) : launch_token<D, kTypeF32, 8>(p, stream);
  if (type == TSD_BF16) return wide ? launch_token<D, kTypeBf16, 16>(p, stream) : launch_token<D, kTypeBf16, 8>(p, stream);
  return wide ? launch_token<D, kTypeE4m3, 16>(p, stream) : launch_token<D, kTypeE4m3, 8>(p, stream);
}

static size_t ticket_bytes() { return (kTokenBlocks * sizeof(unsigned) + 255) / 256 * 256; }

}  // namespace tsd

extern "C" {

size_t tsd_paged_attention_workspace_bytes(const tsd_paged_cache* c, int32_t n_q_heads) {
  if (tsd::check_paged_cache(c) != TSD_OK || n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0) return 0;
  const size_t ht = (size_t)tsd::head_tile(n_q_heads / c->n_kv_heads);
  return tsd::ticket_bytes() + 2 * tsd::kTokenBlocks * (ht * c->head_dim + 2 * ht) * sizeof(float);
}

int tsd_paged_attention(const tsd_paged_cache* c, int32_t n_q_heads, int32_t dtype, const void* q, int64_t q_stride_b,
                        int64_t q_stride_head, const int32_t* kv_lens, void* out, int64_t o_stride_b, int64_t o_stride_head,
                        float* lse, float sm_scale, void* workspace, size_t workspace_bytes, uint32_t* status,
                        tsd_stream_t stream) {
  const int rc = tsd::check_paged_cache(c);
  if (rc != TSD_OK) return rc;
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0 || !q || !out || !(sm_scale == sm_scale)) return TSD_ERR_INVALID_ARG;
  if (dtype != TSD_F32 && dtype != TSD_BF16) return TSD_ERR_UNSUPPORTED;
  if ((dtype == TSD_F32) != (c->dtype == TSD_F32)) return TSD_ERR_UNSUPPORTED;
  if (!tsd::aligned16(q) || !tsd::aligned16(out) || !workspace || !tsd::aligned16(workspace)) return TSD_ERR_INVALID_ARG;
  const int esize = dtype == TSD_F32 ? 4 : 2;
  const int64_t strides[4] = {q_stride_b, o_stride_b, q_stride_head, o_stride_head};
  for (int i = 0; i < 4; ++i)
    if ((i < 2 ? c->batch : n_q_heads) > 1 && (strides[i] < (i == 0 ? 0 : c->head_dim) || (strides[i] * esize) % 16 != 0))
      return TSD_ERR_INVALID_ARG;
  if (workspace_bytes < tsd_paged_attention_workspace_bytes(c, n_q_heads)) return TSD_ERR_WORKSPACE;
  tsd::TokenParams p = {};
  p.cache = tsd::paged_view(*c);
  p.q = q; p.out = out; p.lse = lse; p.lens = kv_lens;
  p.q_b = q_stride_b; p.q_h = q_stride_head; p.o_b = o_stride_b; p.o_h = o_stride_head;
  p.S = c->batch; p.Hq = n_q_heads; p.Hkv = c->n_kv_heads;
  p.group = n_q_heads / c->n_kv_heads;
  const int ht = tsd::head_tile(p.group);
  p.tiles = (p.group + ht - 1) / ht;
  if ((int64_t)p.Hkv * p.tiles > 0x7fffffffll) return TSD_ERR_UNSUPPORTED;
  p.scale_log2e = (float)(sm_scale * 1.4426950408889634);
  p.tickets = static_cast<unsigned*>(workspace);
  p.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + tsd::ticket_bytes());
  p.status = status;
  return c->head_dim == 64 ? tsd::launch_token<64>(c->dtype, p, stream) : tsd::launch_token<128>(c->dtype, p, stream);
}

}  // extern "C"
