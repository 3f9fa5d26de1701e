// Attention of one new token per sequence over a paged K/V cache (no counterpart in the paper, whose passes verify whole blocks:
// tsd_verify_attention).  With q the query rows of the heads that share a kv head,
//     s_t = sm_scale <q, k_t>,   out = sum_t e^(s_t - m) v_t / sum_t e^(s_t - m),   m = max_t s_t.
// Every cached row is read once and used for a few multiply-adds per head, so the kernel is bound by memory; everything in it
// serves to keep loads in flight.
//   split   : the keys of all sequences and heads are laid end to end in chunks of 4 KB of K and 4 KB of V (16 keys of 128 bf16) and cut
//             evenly over the blocks, one per SM, whatever the single lengths are.  Inside a block the warps take the chunks in turn.
//   warp    : a chunk goes from memory straight into the registers of one warp, in the layout that the matrix instruction wants.  For scores,
//             lane (g, t) = (lane / 4, lane % 4) reads 16 bytes of key g at offsets 64 c + 16 t; which dimensions a step of the
//             contraction takes is arbitrary as long as q is laid out alike, so these bytes are the B operand as they are.
//             For the weighted sum, lane (g, t) reads columns 8 g ... of keys 2t, 2t+1, 2t+8, 2t+9 and pairs the keys' halves
//             (one byte permutation per operand register).  K of the next chunk is requested as soon as the scores have used this one's, V likewise.
//   rows    : mma.sync m16n8k16, rows = heads.  Up to 8 heads share a kv head: the other 8 rows carry the residuals of the weights,
//             p - bf16(p), so that the weights count with 16 bits at no cost.  9 to 16 heads: a second product for the residuals.  More: tiles of 16 heads.
//             The tensor memory instructions would bring 128-row tiles, of which 1 to 16 rows would be used, and a trip through shared memory.
//   fp32    : the same loads on CUDA cores (the scores' partial sums of a key meet over its 4 lanes, the weights in shared memory).
//   join    : at the end of a sequence's stretch the warps' running maxima, sums and rows meet in shared memory; a stretch that is not
//             the whole of its sequence goes to the workspace, and the last of its blocks to arrive puts the parts together, in their order.
// Lengths are read on the device: a captured call follows them.  Rows past a length are not loaded.
#include <algorithm>
#include <math_constants.h>
#include "tsd_paged.cuh"

namespace tsd {

constexpr int kTokenBlocks = kPlanSms;  // at most: what the workspace is sized for
constexpr int kMinRounds = 2;           // chunks per warp that a block is worth

enum { kTypeF32 = TSD_F32, kTypeBf16 = TSD_BF16, kTypeE4m3 = TSD_E4M3 };

template <int D, int kType, int HT>
struct TokenPlan {
  static constexpr int kWarps = 8;                                             // two per scheduler: up to 255 registers per thread
  static constexpr int kSize = kType == kTypeF32 ? 4 : kType == kTypeBf16 ? 2 : 1;  // bytes of a cached element
  static constexpr int kRow = D * kSize;                                       // bytes of a row
  static constexpr int kPieces = kRow / 64;                                    // 16-byte pieces per lane and key
  static constexpr int kGroups = 8 / kPieces;                                  // groups of 8 keys per chunk
  static constexpr int kKeys = 8 * kGroups;                                    // keys per chunk
  static constexpr int kSlot = HT * D + 2 * HT;                                // floats of a part in the workspace
  static constexpr int kPitch = D + 4;                                         // floats between rows in shared memory
};

struct TokenParams {
  PagedView cache;
  const void* q;
  void* out;
  float* lse;
  const int32_t* lens;
  int64_t q_b, q_h, o_b, o_h;
  int S, Hq, Hkv, group, tiles;  // tiles: of HT heads per kv head
  float scale_log2e;
  float* parts;        // [2 * blocks] slots: a block's last stretch (even), its first where that began in a block before (odd)
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
// 16 (8) bytes of the cache, or zeros; read once, so L1 keeps nothing of them.
__device__ __forceinline__ uint4 load16(const uint8_t* p, bool wanted) {
  uint4 v;
  asm volatile("{\n.reg .pred w;\nsetp.ne.b32 w, %5, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\nmov.b32 %2, 0;\nmov.b32 %3, 0;\n"
               "@w ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];\n}"
               : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((int)wanted));
  return v;
}
__device__ __forceinline__ uint2 load8(const uint8_t* p, bool wanted) {
  uint2 v;
  asm volatile("{\n.reg .pred w;\nsetp.ne.b32 w, %3, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\n"
               "@w ld.global.nc.L1::no_allocate.v2.b32 {%0, %1}, [%2];\n}"
               : "=&r"(v.x), "=&r"(v.y) : "l"(p), "r"((int)wanted));
  return v;
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two e4m3 codes, in the upper bytes of the two halves of w, as bf16.  Sign, exponent and mantissa move to the places that bf16 has for them;
// the value is then 2^-120 of what the code stands for (its smallest ones a subnormal bf16), and the product with 2^120 is exact.
__device__ __forceinline__ uint32_t widen_e4m3(uint32_t w) {
  const uint32_t x = ((w >> 4) & 0x07f007f0u) | (w & 0x80008000u);
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x7b807b80u));
  return r;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word(const uint2& v, int i) { return i == 0 ? v.x : v.y; }

// Where a chunk lies: sequence, head tile of the sequence, chunk; chunks and keys of the sequence.
struct Cursor {
  int s, hi, c, n, len;
};

template <int D, int kType, int HT>
__global__ void __launch_bounds__(TokenPlan<D, kType, HT>::kWarps * 32, 1) paged_attention_kernel(const TokenParams p) {
  using P = TokenPlan<D, kType, HT>;
  constexpr int NW = P::kWarps, KC = P::kKeys, NG = P::kGroups, NP = P::kPieces;
  constexpr bool kF32 = kType == kTypeF32;
  constexpr int kAcc = kF32 ? HT : D / 8;             // rows of 4 dimensions (fp32), or column blocks of 8
  __shared__ __align__(16) float part_o[NW][8][P::kPitch];
  __shared__ float part_m[NW][8], part_l[NW][8];
  __shared__ __align__(16) float weights[kF32 ? NW : 1][kF32 ? KC : 1][HT];
  __shared__ __align__(16) float q_rows[kF32 ? HT : 1][kF32 ? D : 1];
  __shared__ int last_arrival;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  constexpr unsigned full = 0xffffffffu;
  TokenParams a = p;
  grid_wait(a.cache.k, a.cache.v, a.cache.table, a.q, a.lens, a.cache.k_scale, a.cache.v_scale);
  const int HI = a.Hkv * a.tiles;
  auto length = [&](int s) { return a.lens ? min(max(a.lens[s], 0), a.cache.cap) : a.cache.cap; };
  auto chunks = [&](int len) { return (int)(((unsigned)len + KC - 1) / KC); };

  // ---- this block's share [x0, x1) of all chunks
  int64_t total = 0;
  for (int s = lane; s < a.S; s += 32) {
    const int n = chunks(length(s));
    total += n;
    if (n == 0 && s % (int)gridDim.x == (int)blockIdx.x) {  // a sequence without keys (the lanes of warp 0 write what its rows are)
      if (warp == 0)
        for (int h = 0; h < a.Hq; ++h) {
          if (a.lse) a.lse[(int64_t)s * a.Hq + h] = -CUDART_INF_F;
          uint4* o = reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.out) + (s * a.o_b + h * a.o_h) * (kF32 ? 4 : 2));
          for (int i = 0; i < D * (kF32 ? 4 : 2) / 16; ++i) o[i] = make_uint4(0, 0, 0, 0);
        }
    }
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) total += __shfl_xor_sync(full, total, off);
  total *= HI;
  const int64_t n_blocks = min((int64_t)gridDim.x, (total + NW * kMinRounds - 1) / (NW * kMinRounds));
  if ((int64_t)blockIdx.x >= n_blocks) return;
  // blocks take total / n_blocks chunks each, the first `more` of them one more
  const int64_t each = total / n_blocks, more = total % n_blocks;
  auto first_of = [&](int64_t b) { return b * each + min(b, more); };
  auto block_of = [&](int64_t x) { return x < more * (each + 1) ? x / (each + 1) : more + (x - more * (each + 1)) / each; };
  const int64_t x0 = first_of(blockIdx.x), x1 = first_of(blockIdx.x + 1);

  // ---- where chunk x0 lies
  Cursor seg;  // of the block's stretch at hand
  int64_t seg_first;  // first chunk of its (sequence, head tile)
  {
    int64_t before = 0;
    seg.s = a.S;
    for (int s0 = 0; s0 < a.S; s0 += 32) {
      const int len = s0 + lane < a.S ? length(s0 + lane) : 0;
      const int64_t mine = (int64_t)chunks(len) * HI;
      int64_t upto = mine;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int64_t o = __shfl_up_sync(full, upto, off);
        if (lane >= off) upto += o;
      }
      const unsigned hit = __ballot_sync(full, before + upto > x0);
      if (hit) {
        const int l = __ffs(hit) - 1;
        seg.s = s0 + l;
        seg.len = __shfl_sync(full, len, l);
        before += __shfl_sync(full, upto - mine, l);
        break;
      }
      before += __shfl_sync(full, upto, 31);
    }
    seg.n = chunks(seg.len);
    seg.hi = (int)((x0 - before) / seg.n);
    seg.c = (int)((x0 - before) % seg.n);
    seg_first = x0 - seg.c;
  }
  auto next_sequence = [&](Cursor& cur) {
    cur.hi = 0;
    do {
      if (++cur.s >= a.S) {  // behind the last chunk: never loaded
        cur.n = 0x7fffffff;
        cur.len = 0;
        return;
      }
      cur.len = length(cur.s);
      cur.n = chunks(cur.len);
    } while (cur.n == 0);
  };
  auto advance = [&](Cursor& cur, int step) {
    cur.c += step;
    while (cur.c >= cur.n) {
      cur.c -= cur.n;
      if (++cur.hi == HI) next_sequence(cur);
    }
  };

  bool bad_page = false;
  const int row_mask = (1 << a.cache.shift) - 1;
  // lane l < NG: the page of the chunk's keys [8 l, 8 l + 8), or -1
  auto pages_of = [&](const Cursor& cur) {
    const int key = cur.c * KC + 8 * lane;
    int page = -1;
    if (lane < NG && key < cur.len) {
      page = page_of(a.cache, cur.s, key);
      if (page < 0) bad_page = true;
    }
    return page;
  };
  uint4 kr[8];
  uint4 vr[8];
  const int64_t row_bytes = a.cache.ps_r * P::kSize;
  auto load_k = [&](const Cursor& cur, int pages) {
    const int key0 = cur.c * KC;
    const uint8_t* base = static_cast<const uint8_t*>(a.cache.k) + (cur.hi / a.tiles) * (a.cache.ps_h * P::kSize) + 16 * t;
#pragma unroll
    for (int nb = 0; nb < NG; ++nb) {
      const int page = __shfl_sync(full, pages, nb), key = key0 + 8 * nb + g;
      const uint8_t* row = base + (int64_t)page * (a.cache.ps_p * P::kSize) + (key & row_mask) * row_bytes;
#pragma unroll
      for (int c = 0; c < NP; ++c) kr[nb * NP + c] = load16(row + 64 * c, page >= 0 && key < cur.len);
    }
  };
  // bf16 and e4m3: keys 16 sub + {2t, 2t+1, 2t+8, 2t+9}; fp32: whole rows, a warp (or half of one) per key
  auto load_v = [&](const Cursor& cur, int pages) {
    const int key0 = cur.c * KC;
    const uint8_t* base = static_cast<const uint8_t*>(a.cache.v) + (cur.hi / a.tiles) * (a.cache.ps_h * P::kSize);
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int in = D == 128 ? i : 2 * i + (lane >> 4), key = key0 + in;
        const int page = __shfl_sync(full, pages, in >> 3);
        vr[i] = load16(base + (int64_t)page * (a.cache.ps_p * 4) + (key & row_mask) * row_bytes + 16 * (D == 128 ? lane : lane & 15),
                       page >= 0 && key < cur.len);
      }
    } else {
#pragma unroll
      for (int nb = 0; nb < NG; ++nb) {  // 8 keys: two of them are this lane's
        const int page = __shfl_sync(full, pages, nb), key = key0 + 8 * nb + 2 * t;
        const uint8_t* row = base + (int64_t)page * (a.cache.ps_p * P::kSize) + (key & row_mask) * row_bytes;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool wanted = page >= 0 && key + e < cur.len;
          if constexpr (P::kRow == 64) {  // e4m3, 64 dimensions: 8 bytes; the lane's keys of a group share a register quadruple
            const uint2 v = load8(row + e * row_bytes + 8 * g, wanted);
            (e ? vr[nb].z : vr[nb].x) = v.x;
            (e ? vr[nb].w : vr[nb].y) = v.y;
          } else {
#pragma unroll
            for (int c = 0; c < P::kRow / 128; ++c)
              vr[(nb * 2 + e) * (P::kRow / 128) + c] = load16(row + e * row_bytes + 128 * c + 16 * g, wanted);
          }
        }
      }
    }
  };
  // the lane's part of the query rows of a (sequence, head tile)
  uint32_t qr[kF32 ? 1 : D / 8], qr8[kF32 || HT == 8 ? 1 : D / 8];
  float score_scale = 0.f;
  auto load_q = [&](const Cursor& cur) {
    const int kv = cur.hi / a.tiles, h0 = kv * a.group + (cur.hi % a.tiles) * HT, rows = min(HT, (kv + 1) * a.group - h0);
    score_scale = a.scale_log2e * (kType == kTypeE4m3 && a.cache.k_scale ? a.cache.k_scale[kv] : 1.f);
    if constexpr (kF32) {
      for (int i = tid; i < HT * D; i += NW * 32)
        q_rows[i / D][i % D] = i / D < rows ? static_cast<const float*>(a.q)[cur.s * a.q_b + (h0 + i / D) * a.q_h + i % D] : 0.f;
    } else {
      constexpr int E = 16 / P::kSize;  // elements of a lane's piece
      auto load_row = [&](int r, uint32_t* to) {
        const __nv_bfloat16* row = static_cast<const __nv_bfloat16*>(a.q) + cur.s * a.q_b + (int64_t)(h0 + r) * a.q_h;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
          for (int e = 0; e < E / 8; ++e) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < rows) v = *reinterpret_cast<const uint4*>(row + c * 4 * E + t * E + e * 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) to[(c * (E / 8) + e) * 4 + i] = word(v, i);
          }
      };
      load_row(g, qr);
      if constexpr (HT == 16) load_row(g + 8, qr8);
    }
  };

  float acc[kAcc][4];
  float m[HT == 16 && !kF32 ? 2 : 1], l[HT == 16 && !kF32 ? 2 : 1];  // fp32: of row lane % HT, equal in the lanes that share it

  // ---- the warp's first chunk
  Cursor nxt = seg;
  advance(nxt, warp);
  int64_t x = x0 + warp;  // the chunk in kr and vr
  int pages = x < x1 ? pages_of(nxt) : -1;
  if (x < x1) {
    load_k(nxt, pages);
    load_v(nxt, pages);
  }
  Cursor cur = nxt;
  advance(nxt, NW);
  pages = x + NW < x1 ? pages_of(nxt) : -1;
  load_q(seg);
  if constexpr (kF32) __syncthreads();

  for (int64_t pos = x0; pos < x1;) {
    const int64_t seg_end = min(x1, seg_first + seg.n);
    const int kv = seg.hi / a.tiles, h0 = kv * a.group + (seg.hi % a.tiles) * HT, rows = min(HT, (kv + 1) * a.group - h0);
#pragma unroll
    for (int i = 0; i < kAcc; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(m) / 4); ++i) { m[i] = -CUDART_INF_F; l[i] = 0.f; }

    for (; x < seg_end; x += NW) {
      const int left = cur.len - cur.c * KC;  // keys of the chunk that count: 1 and up
      const bool more_chunks = x + NW < x1;
      if constexpr (!kF32) {
        // ---------------------------------------------------------------- scores
        float sc[NG][4];
#pragma unroll
        for (int nb = 0; nb < NG; ++nb) {
          sc[nb][0] = sc[nb][1] = sc[nb][2] = sc[nb][3] = 0.f;
#pragma unroll
          for (int c = 0; c < NP; ++c) {
            const uint4 kw = kr[nb * NP + c];
            if constexpr (kType == kTypeBf16) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int w = c * 4 + 2 * e;
                mma(sc[nb], qr[w], HT == 16 ? qr8[w % (D / 8)] : 0u, qr[w + 1], HT == 16 ? qr8[(w + 1) % (D / 8)] : 0u, word(kw, 2 * e), word(kw, 2 * e + 1));
              }
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int w = c * 8 + 2 * e;
                mma(sc[nb], qr[w], HT == 16 ? qr8[w] : 0u, qr[w + 1], HT == 16 ? qr8[w + 1] : 0u,
                    widen_e4m3(__byte_perm(word(kw, e), 0, 0x1100)), widen_e4m3(__byte_perm(word(kw, e), 0, 0x3322)));
              }
            }
          }
        }
        if (more_chunks) load_k(nxt, pages);
        // ---------------------------------------------------------------- weights
        constexpr int NR = HT / 8;
        float alpha[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          float top = -CUDART_INF_F;
#pragma unroll
          for (int nb = 0; nb < NG; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& z = sc[nb][2 * r + e];
              z = 8 * nb + 2 * t + e < left ? z * score_scale : -CUDART_INF_F;
              top = fmaxf(top, z);
            }
          top = fmaxf(top, __shfl_xor_sync(full, top, 1));
          top = fmaxf(top, __shfl_xor_sync(full, top, 2));
          const float m_new = fmaxf(m[r], top);
          alpha[r] = exp2_approx(m[r] - m_new);
          m[r] = m_new;
          float sum = 0.f;
#pragma unroll
          for (int nb = 0; nb < NG; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& z = sc[nb][2 * r + e];
              z = exp2_approx(z - m_new);
              sum += z;
            }
          l[r] = fmaf(l[r], alpha[r], sum);
        }
        bool moved = alpha[0] != 1.f;
        if (NR == 2) moved |= alpha[NR - 1] != 1.f;
        if (__any_sync(full, moved)) {
#pragma unroll
          for (int i = 0; i < kAcc; ++i) {
            acc[i][0] *= alpha[0]; acc[i][1] *= alpha[0];
            acc[i][2] *= alpha[NR - 1]; acc[i][3] *= alpha[NR - 1];
          }
        }
        // ---------------------------------------------------------------- weighted sum of the values
#pragma unroll
        for (int sub = 0; sub < NG / 2; ++sub) {
          float* w0 = sc[2 * sub];
          float* w1 = sc[2 * sub + 1];
          const uint32_t a0 = bf16_pair(w0[0], w0[1]), a2 = bf16_pair(w1[0], w1[1]);
          auto rest = [](uint32_t hi, float x, float y) {  // what the bf16 pair leaves of (x, y)
            return bf16_pair(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u));
          };
          const uint32_t r0 = rest(a0, w0[0], w0[1]), r2 = rest(a2, w1[0], w1[1]);
          uint32_t a1 = r0, a3 = r2, r1 = 0, r3 = 0;
          if constexpr (HT == 16) {
            a1 = bf16_pair(w0[2], w0[3]);
            a3 = bf16_pair(w1[2], w1[3]);
            r1 = rest(a1, w0[2], w0[3]);
            r3 = rest(a3, w1[2], w1[3]);
          }
          auto step = [&](float (&o)[4], uint32_t b0, uint32_t b1) {
            mma(o, a0, a1, a2, a3, b0, b1);
            if constexpr (HT == 16) mma(o, r0, r1, r2, r3, b0, b1);
          };
          if constexpr (kType == kTypeBf16) {
            constexpr int H2 = D / 64;
#pragma unroll
            for (int h2 = 0; h2 < H2; ++h2) {
              const uint4 &u0 = vr[(sub * 4 + 0) * H2 + h2], &u1 = vr[(sub * 4 + 1) * H2 + h2], &u2 = vr[(sub * 4 + 2) * H2 + h2],
                          &u3 = vr[(sub * 4 + 3) * H2 + h2];
#pragma unroll
              for (int j = 0; j < 8; ++j)
                step(acc[h2 * 8 + j], __byte_perm(word(u0, j >> 1), word(u1, j >> 1), j & 1 ? 0x7632 : 0x5410),
                     __byte_perm(word(u2, j >> 1), word(u3, j >> 1), j & 1 ? 0x7632 : 0x5410));
            }
          } else {
            // byte j of the keys' words into the upper bytes of the halves
            constexpr uint32_t pick[4] = {0x4400, 0x5511, 0x6622, 0x7733};
#pragma unroll
            for (int j = 0; j < D / 8; ++j) {
              uint32_t x0w, x1w, x2w, x3w;
              if constexpr (P::kRow == 64) {
                const uint4 &u = vr[2 * sub], &v = vr[2 * sub + 1];
                x0w = word(u, j >> 2); x1w = word(u, 2 + (j >> 2)); x2w = word(v, j >> 2); x3w = word(v, 2 + (j >> 2));
              } else {
                x0w = word(vr[sub * 4], j >> 2); x1w = word(vr[sub * 4 + 1], j >> 2);
                x2w = word(vr[sub * 4 + 2], j >> 2); x3w = word(vr[sub * 4 + 3], j >> 2);
              }
              step(acc[j], widen_e4m3(__byte_perm(x0w, x1w, pick[j & 3])), widen_e4m3(__byte_perm(x2w, x3w, pick[j & 3])));
            }
          }
        }
        if (more_chunks) load_v(nxt, pages);
      } else {
        // ---------------------------------------------------------------- fp32 scores: 4 lanes per key
        float mine[NG];  // of row lane % HT: keys
#pragma unroll
        for (int nb = 0; nb < NG; ++nb) mine[nb] = 0.f;
#pragma unroll
        for (int r = 0; r < HT; ++r) {
          if (r < rows) {
#pragma unroll
            for (int nb = 0; nb < NG; ++nb) {
              float z = 0.f;
#pragma unroll
              for (int c = 0; c < NP; ++c) {
                const float4 qv = *reinterpret_cast<const float4*>(&q_rows[r][16 * c + 4 * t]);
                const uint4 kw = kr[nb * NP + c];
                z = fmaf(qv.x, __uint_as_float(kw.x), z);
                z = fmaf(qv.y, __uint_as_float(kw.y), z);
                z = fmaf(qv.z, __uint_as_float(kw.z), z);
                z = fmaf(qv.w, __uint_as_float(kw.w), z);
              }
              z += __shfl_xor_sync(full, z, 1);
              z += __shfl_xor_sync(full, z, 2);
              if (t == 0) weights[warp][8 * nb + g][r] = 8 * nb + g < left ? z * score_scale : -CUDART_INF_F;
            }
          }
        }
        if (more_chunks) load_k(nxt, pages);
        __syncwarp();
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
#pragma unroll
          for (int off = HT; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(full, top, off));
          const float m_new = fmaxf(m[0], top), alpha = exp2f(m[0] - m_new);
          m[0] = m_new;
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < KC / KL; ++i) {
            z[i] = exp2f(z[i] - m_new);
            sum += z[i];
            weights[warp][i * KL + lane / HT][r] = z[i];
          }
#pragma unroll
          for (int off = HT; off < 32; off <<= 1) sum += __shfl_xor_sync(full, sum, off);
          l[0] = fmaf(l[0], alpha, sum);
          if (__any_sync(full, alpha != 1.f)) {
#pragma unroll
            for (int i = 0; i < HT; ++i) {
              const float f = __shfl_sync(full, alpha, i);
              acc[i][0] *= f; acc[i][1] *= f; acc[i][2] *= f; acc[i][3] *= f;
            }
          }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int in = D == 128 ? i : 2 * i + (lane >> 4);
          const float4 v = make_float4(__uint_as_float(vr[i].x), __uint_as_float(vr[i].y), __uint_as_float(vr[i].z), __uint_as_float(vr[i].w));
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
        if (more_chunks) load_v(nxt, pages);
        __syncwarp();
      }
      cur = nxt;
      advance(nxt, NW);
      pages = x + 2 * NW < x1 ? pages_of(nxt) : -1;
    }

    // ---- the stretch ends: what the warps hold meets in shared memory, 8 rows at a time
    const Cursor done = seg;
    const int64_t done_first = seg_first;
    advance(seg, (int)(seg_end - pos));  // the next stretch; its queries are requested before the barriers below
    seg_first = seg_end;                 // (a stretch that does not end its sequence is the block's last)
    if constexpr (!kF32)
      if (seg_end < x1) load_q(seg);
    const bool whole = done_first >= x0 && done_first + done.n <= x1;
    const bool begins_before = done_first < x0;
    const int64_t b_first = whole ? 0 : block_of(done_first);
    const float v_scale = kType == kTypeE4m3 && a.cache.v_scale ? a.cache.v_scale[kv] : 1.f;
    float* slot = a.parts + (2 * (int64_t)blockIdx.x + (begins_before ? 1 : 0)) * P::kSlot;

    // rows [8 half, 8 half + 8) of all warps -> the sequence's output, or the block's part in the workspace
    auto meet = [&](int half, bool final) {
      __syncthreads();
      for (int e = tid; e < min(8, rows - 8 * half) * (D / 4); e += NW * 32) {
        const int r = e / (D / 4), col = 4 * (e % (D / 4));
        float top = part_m[0][r];
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, part_m[w][r]);
        float sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float mw = part_m[w][r];
          if (mw == -CUDART_INF_F) continue;  // a warp without a chunk
          const float f = exp2f(mw - top);
          const float4 v = *reinterpret_cast<const float4*>(&part_o[w][r][col]);
          sum = fmaf(part_l[w][r], f, sum);
          o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
        }
        const int row = 8 * half + r;
        if (final) {
          const float f = v_scale / sum;
          const int64_t to = done.s * a.o_b + (int64_t)(h0 + row) * a.o_h + col;
          if constexpr (kF32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to) = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
          else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to) = make_uint2(bf16_pair(o.x * f, o.y * f), bf16_pair(o.z * f, o.w * f));
          if (a.lse && col == 0) a.lse[(int64_t)done.s * a.Hq + h0 + row] = (top + log2f(sum)) * 0.6931471805599453f;
        } else {
          *reinterpret_cast<float4*>(slot + row * D + col) = o;
          if (col == 0) { slot[HT * D + row] = top; slot[HT * D + HT + row] = sum; }
        }
      }
      __syncthreads();
    };
#pragma unroll
    for (int half = 0; half < HT / 8; ++half) {
      if (8 * half >= rows) break;
      if constexpr (kF32) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          float(&o)[4] = acc[8 * half + r];
          if (D == 64) {  // the two halves of the warp had different keys
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += __shfl_xor_sync(full, o[i], 16);
          }
          if (8 * half + r < rows && (D == 128 || lane < 16)) *reinterpret_cast<float4*>(&part_o[warp][r][4 * lane]) = make_float4(o[0], o[1], o[2], o[3]);
        }
        if (lane >= 8 * half && lane < 8 * half + 8) { part_m[warp][lane - 8 * half] = m[0]; part_l[warp][lane - 8 * half] = l[0]; }
      } else {
        float sum = l[HT == 16 ? half : 0];
        sum += __shfl_xor_sync(full, sum, 1);
        sum += __shfl_xor_sync(full, sum, 2);
        if (t == 0) { part_m[warp][g] = m[HT == 16 ? half : 0]; part_l[warp][g] = sum; }
        if (8 * half + g < rows) {
          constexpr int kRun = P::kSize == 1 && D == 128 ? 16 : 8;  // columns of a lane in a row, per run
#pragma unroll
          for (int i = 0; i < kAcc / kRun; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int j = 0; j < kRun; j += 4) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float(&o)[4] = acc[i * kRun + j + k];
                  v[k] = HT == 16 ? o[2 * half + e] : o[e] + o[2 + e];
                }
                *reinterpret_cast<float4*>(&part_o[warp][g][i * 64 + (2 * t + e) * kRun + j]) = make_float4(v[0], v[1], v[2], v[3]);
              }
        }
      }
      meet(half, whole);
    }
    if (!whole) {
      // The part is in the workspace.  The last of the sequence's blocks to arrive puts all parts together.
      const int64_t b_last = block_of(done_first + done.n - 1);
      const int n_parts = (int)(b_last - b_first) + 1;
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        last_arrival = atomicAdd(a.tickets + b_first, 1u) + 1u == (unsigned)n_parts;
        if (last_arrival) a.tickets[b_first] = 0;
        __threadfence();
      }
      __syncthreads();
      if (last_arrival) {
        auto part_at = [&](int i) { return a.parts + (2 * (b_first + i) + (i ? 1 : 0)) * P::kSlot; };
#pragma unroll 1
        for (int half = 0; half < HT / 8; ++half) {
          if (8 * half >= rows) break;
          // this warp's parts: warp, warp + NW, ...; lane = (part in a group of 4, row)
          constexpr int kRounds = (kTokenBlocks + 4 * NW - 1) / (4 * NW);
          float pm[kRounds], top = -CUDART_INF_F, sum = 0.f;
          const int r = lane & 7;
          const bool row_ok = 8 * half + r < rows;
#pragma unroll
          for (int k = 0; k < kRounds; ++k) {
            const int i = warp + NW * (4 * k + (lane >> 3));
            pm[k] = i < n_parts && row_ok ? __ldcg(part_at(i) + HT * D + 8 * half + r) : -CUDART_INF_F;
            top = fmaxf(top, pm[k]);
          }
          top = fmaxf(top, __shfl_xor_sync(full, top, 8));
          top = fmaxf(top, __shfl_xor_sync(full, top, 16));
#pragma unroll
          for (int k = 0; k < kRounds; ++k) {
            const int i = warp + NW * (4 * k + (lane >> 3));
            const bool there = i < n_parts && row_ok;
            pm[k] = there ? exp2f(pm[k] - top) : 0.f;
            if (there) sum = fmaf(__ldcg(part_at(i) + HT * D + HT + 8 * half + r), pm[k], sum);
          }
          sum += __shfl_xor_sync(full, sum, 8);
          sum += __shfl_xor_sync(full, sum, 16);
          if (lane < 8) { part_m[warp][lane] = top; part_l[warp][lane] = sum; }
          constexpr int kVec = 8 * D / 128;  // float4 of the 8 rows, per lane
#pragma unroll
          for (int v = 0; v < kVec; ++v) {
            const int e = lane + 32 * v, vr_ = e / (D / 4), col = 4 * (e % (D / 4));
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            if (8 * half + (32 * v) / (D / 4) >= rows) break;
#pragma unroll
            for (int k = 0; k < kRounds; ++k)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const int i = warp + NW * (4 * k + q);
                const float f = __shfl_sync(full, pm[k], q * 8 + vr_);
                if (i < n_parts && 8 * half + vr_ < rows) {
                  const float4 x4 = __ldcg(reinterpret_cast<const float4*>(part_at(i) + (8 * half + vr_) * D + col));
                  o.x = fmaf(x4.x, f, o.x); o.y = fmaf(x4.y, f, o.y); o.z = fmaf(x4.z, f, o.z); o.w = fmaf(x4.w, f, o.w);
                }
              }
            *reinterpret_cast<float4*>(&part_o[warp][vr_][col]) = o;
          }
          meet(half, true);
        }
      }
    }
    if constexpr (kF32) {
      if (seg_end < x1) {
        load_q(seg);
        __syncthreads();
      }
    }
    pos = seg_end;
  }
  if (__any_sync(full, bad_page) && lane == 0 && a.status) atomicOr(a.status, TSD_STATUS_BAD_INDEX);
}

// Heads per tile: 8 where they suffice (the residuals then ride in the other 8 rows of a product).
static int head_tile(int group) { return group <= 8 ? 8 : 16; }

template <int D, int kType, int HT>
static int launch_token(const TokenParams& p, cudaStream_t stream) {
  using P = TokenPlan<D, kType, HT>;
  const int64_t most = (int64_t)p.S * p.Hkv * p.tiles * ((p.cache.cap + P::kKeys - 1) / P::kKeys);  // chunks, if every sequence were full
  const int64_t grid = std::min<int64_t>(kTokenBlocks, (most + P::kWarps * kMinRounds - 1) / (P::kWarps * kMinRounds));
  const cudaError_t e = launch(paged_attention_kernel<D, kType, HT>, dim3((unsigned)std::max<int64_t>(grid, 1)), dim3(P::kWarps * 32), 0, stream, p);
  return e != cudaSuccess ? cuda_fail(e, "paged_attention_kernel") : TSD_OK;
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
    if ((i < 2 ? c->batch : n_q_heads) > 1 && (strides[i] < (i < 2 ? 0 : c->head_dim) || (strides[i] * esize) % 16 != 0))
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
