// Attention of one new token over the pages of a paged cache.
//
//     x_i = scale * q . K[i]  (capped: c tanh(x / c)),   out = sum_i e^(x_i - m) V[i] / sum_i e^(x_i - m)
//
// One pass over the rows with a running maximum m and sum, logits in the base-2 domain.  All query heads of a KV
// head's group share the read of its rows.  What has to be read is the rows, once; everything else is small, so the
// kernel is built to keep copies in flight:
//
// The tiles of all heads (64 rows; 32 of 512 bytes) form one line, which is cut into equal parts, one per CTA, two
// CTAs per SM: heads of any lengths load all SMs alike.  Row counts live on the device, so every CTA finds its part
// itself.  A producer warp walks the part: it looks up the tile's pages and has TMA fetch K and V in boxes of 16 rows
// (the least page) into a ring of stages; boxes behind a head's last row are not fetched.  Four warps consume a
// tile, a quarter of its rows each, with maxima and sums of their own until the head or the part ends; then they meet
// through the memory of the last stage.  A head inside one part is finished there.  Of a head that continues in other
// parts the partial result goes to memory; the CTA that comes last, as a counter tells, joins them in order.
//
// bf16: S = Q K^T and O += P V by mma.sync m16n8k16 (2 % of the tensor peak at the rate of HBM).  With up to 8 queries
// the other 8 rows of the A operand are free: they carry what rounding the probabilities to bf16 left over, so the
// products with V keep 16 bits of every probability at no cost; with 9 to 16 queries a second product does.  More
// queries per KV head than 16 are taken 16 at a time.  fp32: a lane has a row (or a half or quarter of it) for the
// logits, and some columns for the product with V; up to 8 queries at a time.
#include <algorithm>
#include <type_traits>

#include <math.h>

#include "sm100_ptx.cuh"

namespace lava {
namespace {

using namespace sm100;

constexpr int kConsumers = 4;                  // warps
constexpr int kThreads = (kConsumers + 1) * 32;
constexpr int kBoxRows = 16;
constexpr int kCtasPerSm = 2;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int D, bool BF16, int Q>
struct Shape {
  static constexpr int kRowBytes = D * (BF16 ? 2 : 4);
  static constexpr int kTile = kRowBytes == 512 ? 32 : 64;       // rows
  static constexpr int kWarpRows = kTile / kConsumers;
  static constexpr int kBoxBytes = kBoxRows * kRowBytes;
  static constexpr int kTileBytes = kTile * kRowBytes;
  static constexpr int kStageBytes = 2 * kTileBytes;             // K, V
  static constexpr int kStages = 96 * 1024 / kStageBytes;
  static constexpr int kSmem = kStages * kStageBytes + 1024;     // (aligned to the swizzle's period inside)
  static_assert(kConsumers * Q * D * 4 <= kStageBytes, "the warps' results fit a stage");
  static constexpr int kSmall = 128 * 1024 / kStageBytes, kLarge = 2 * kSmall;  // tiles of a piece
};

struct PageParams {
  Cache c;
  int first_head;          // of the call's first layer
  int heads;               // of the call's layers
  int subs, per_sub;       // a group's queries are taken in `subs` portions of `per_sub`
  const void* q;           // [layers, batch, H_q, d]
  const int* table;
  const int* rows;
  void* out;
  float* lse;
  float* part;             // [CTA][2][Q][D]: partial results of the part's first and last head,
  float2* part_ml;         // [CTA][2][Q]: the maximum that they are relative to, and the sum
  int* counters;           // [CTA]: parts that have left their result of the head that begins last in CTA's part
  unsigned* status;
  long long wait_cycles;
};

struct Ctl {
  volatile int abort_flag;
  long long wait_cycles;
};

struct Start {
  int head, sub, tile;     // head of the call, portion of its queries, tile
  int end, first, pieces;  // a piece of a portion: its last tile + 1, the portion's first piece and their number
};

// Sums over heads (the host has seen to it that they fit).
struct Counts {
  int tiles, boxes, small, large;  // tiles, boxes of 16 rows, pieces of both sizes
  int most;                        // boxes of the longest head
  __device__ __forceinline__ void add(const Counts& y) {
    tiles += y.tiles;
    boxes += y.boxes;
    small += y.small;
    large += y.large;
    most = max(most, y.most);
  }
};

template <class S>
__device__ __forceinline__ int tiles_of(int len) {
  return (len + S::kTile - 1) / S::kTile;
}
__device__ __forceinline__ int head_len(const PageParams& p, int h) {
  return min(max(0, p.rows[p.first_head + h]), p.c.max_pages << p.c.page_shift);
}

// Byte address of 16-byte piece c of row r in a tile: boxes of 16 rows, in them blocks of 128 bytes of every row
// with the 128-byte swizzle.
template <class S>
__device__ __forceinline__ uint32_t piece_at(uint32_t tile, int r, int c) {
  return tile + (r >> 4) * S::kBoxBytes + (c >> 3) * (kBoxRows * 128) + (r & 15) * 128 + (((c ^ r) & 7) << 4);
}

// The logit in the base-2 domain of a product of q and a row.
struct Logit {
  float scale, in, cap;  // scale * log2(e); or, capped: scale / cap, cap * log2(e)
  __device__ explicit Logit(const Cache& c)
      : scale(c.scale * kLog2e), in(c.softcap > 0.f ? c.scale / c.softcap : 0.f), cap(c.softcap * kLog2e) {}
  __device__ __forceinline__ float of(float s) const {
    if (cap == 0.f) return s * scale;
    // tanh z = 1 - 2 / (e^(2 z) + 1); near zero, where that cancels, its series (to z^9: 2e-9 at 1/4)
    const float z = s * in, zz = z * z;
    const float t = 1.f - __fdividef(2.f, fast_exp2(z * (2.f * kLog2e)) + 1.f);
    const float series = z * fmaf(zz, fmaf(zz, fmaf(zz, fmaf(zz, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return cap * (fabsf(z) < 0.25f ? series : t);
  }
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ void ldmatrix_x4(uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3, uint32_t saddr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(saddr)
               : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// barrier of the consumer warps; whether `x` holds in all their threads
__device__ __forceinline__ bool meet_all(bool x) {
  uint32_t y;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbarrier.cta.red.and.pred p, 1, 128, q;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(y) : "r"((uint32_t)x) : "memory");
  return y != 0;
}
static_assert(kConsumers * 32 == 128, "meet_all");
__device__ __forceinline__ void meet() { named_bar_sync(1, kConsumers * 32); }
// what exponentials are taken against: 0 where there is no logit above -infinity
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

// largest logit of query q that the warps have met
template <int Q>
__device__ __forceinline__ float top_of(const float2 (*stats)[Q], int q) {
  float top = stats[0][q].x;
#pragma unroll
  for (int i = 1; i < kConsumers; ++i) top = fmaxf(top, stats[i][q].x);
  return top;
}

// ---- bf16: tensor cores ----------------------------------------------------------------------------
// Thread (g = lane / 4, t = lane % 4) has query row g, and with 16 queries g + 8 too.
template <int D, int Q>
struct TensorWarp {
  using S = Shape<D, true, Q>;
  static constexpr int kRowsOf = Q / 8;
  static constexpr bool kOwnQueries = true;
  uint32_t qa[D / 16][2 * kRowsOf];
  float m[kRowsOf], l[kRowsOf], o[D / 8][4];

  __device__ __forceinline__ void begin(const PageParams& p, size_t q_row, int queries) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
    for (int u = 0; u < kRowsOf; ++u) {
      const bool there = g + 8 * u < queries;
      const uint32_t* qh = reinterpret_cast<const uint32_t*>(p.q) + (q_row + g + 8 * u) * (D / 2);
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        qa[s][u] = there ? qh[8 * s + t] : 0u;
        qa[s][kRowsOf + u] = there ? qh[8 * s + 4 + t] : 0u;
      }
      m[u] = -INFINITY;
      l[u] = 0.f;
    }
#pragma unroll
    for (int nd = 0; nd < D / 8; ++nd) o[nd][0] = o[nd][1] = o[nd][2] = o[nd][3] = 0.f;
  }

  // rows r0 ... r0 + 15 of the tile, of which `valid` (> 0) are there; v_ready() waits for V
  template <class Wait>
  __device__ __forceinline__ bool tile(uint32_t k_tile, uint32_t v_tile, int r0, int valid, const Logit& logit, float*,
                                       Wait v_ready) {
    const int lane = threadIdx.x & 31, t = lane & 3, mi = lane >> 3, r8 = lane & 7;
    float s[2][4] = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {  // matrices (keys 0-7, piece 2 ks), (0-7, 2 ks + 1), (8-15, ...)
      uint32_t b0, b1, b2, b3;
      ldmatrix_x4(b0, b1, b2, b3, piece_at<S>(k_tile, r0 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1)));
      const uint32_t a0 = qa[ks][0], a1 = kRowsOf == 2 ? qa[ks][1] : 0u;
      const uint32_t a2 = qa[ks][kRowsOf], a3 = kRowsOf == 2 ? qa[ks][kRowsOf + 1] : 0u;
      mma_bf16_16816(s[0][0], s[0][1], s[0][2], s[0][3], a0, a1, a2, a3, b0, b1);
      mma_bf16_16816(s[1][0], s[1][1], s[1][2], s[1][3], a0, a1, a2, a3, b2, b3);
    }
    uint32_t hi[2][kRowsOf], lo[2][kRowsOf];  // [keys 0-7, 8-15][row]
    float corr[kRowsOf];
    bool moved = false;
#pragma unroll
    for (int u = 0; u < kRowsOf; ++u) {
      float x[2][2], best = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[n][e] = 8 * n + 2 * t + e < valid ? logit.of(s[n][2 * u + e]) : -INFINITY;
          best = fmaxf(best, x[n][e]);
        }
      best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 1));
      best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 2));
      const float m_new = fmaxf(m[u], best), ref = finite_ref(m_new);
      corr[u] = fast_exp2(m[u] - ref);
      moved |= m_new != m[u];
      m[u] = m_new;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        x[n][0] = fast_exp2(x[n][0] - ref);
        x[n][1] = fast_exp2(x[n][1] - ref);
        hi[n][u] = pack_bf16(x[n][0], x[n][1]);
        lo[n][u] = pack_bf16(x[n][0] - bf16_lo(hi[n][u]), x[n][1] - bf16_hi(hi[n][u]));
      }
      l[u] = fmaf(l[u], corr[u], (x[0][0] + x[0][1]) + (x[1][0] + x[1][1]));
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int nd = 0; nd < D / 8; ++nd)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nd][e] *= corr[kRowsOf == 2 ? e >> 1 : 0];
    }
    if (!v_ready()) return false;
    if (valid < 16) {  // rows behind the last one may hold anything: their probabilities are 0, so must they be
      for (int i = lane; i < (16 - valid) * (D / 8); i += 32)
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(piece_at<S>(v_tile, r0 + valid + i / (D / 8), i % (D / 8))),
                     "r"(0) : "memory");
      fence_async_proxy();  // (before the next copy into this stage)
      __syncwarp();
    }
#pragma unroll
    for (int nd = 0; nd < D / 8; nd += 2) {
      uint32_t b0, b1, b2, b3;
      ldmatrix_x4_trans(b0, b1, b2, b3, piece_at<S>(v_tile, r0 + (mi & 1) * 8 + r8, nd + (mi >> 1)));
      if constexpr (kRowsOf == 1) {
        mma_bf16_16816(o[nd][0], o[nd][1], o[nd][2], o[nd][3], hi[0][0], lo[0][0], hi[1][0], lo[1][0], b0, b1);
        mma_bf16_16816(o[nd + 1][0], o[nd + 1][1], o[nd + 1][2], o[nd + 1][3], hi[0][0], lo[0][0], hi[1][0], lo[1][0], b2, b3);
      } else {
        mma_bf16_16816(o[nd][0], o[nd][1], o[nd][2], o[nd][3], lo[0][0], lo[0][1], lo[1][0], lo[1][1], b0, b1);
        mma_bf16_16816(o[nd + 1][0], o[nd + 1][1], o[nd + 1][2], o[nd + 1][3], lo[0][0], lo[0][1], lo[1][0], lo[1][1], b2, b3);
        mma_bf16_16816(o[nd][0], o[nd][1], o[nd][2], o[nd][3], hi[0][0], hi[0][1], hi[1][0], hi[1][1], b0, b1);
        mma_bf16_16816(o[nd + 1][0], o[nd + 1][1], o[nd + 1][2], o[nd + 1][3], hi[0][0], hi[0][1], hi[1][0], hi[1][1], b2, b3);
      }
    }
    return true;
  }

  __device__ __forceinline__ void leave_stats(float2* ml) {  // [Q] of this warp
    const int g = (threadIdx.x & 31) >> 2;
#pragma unroll
    for (int u = 0; u < kRowsOf; ++u) {
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 1);
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 2);
      if ((threadIdx.x & 3) == 0) ml[g + 8 * u] = make_float2(m[u], l[u]);
    }
  }
  // column `col` of query q lies at float `col ^ swizzle(q)` of its row (spreads the rows over the banks)
  static __device__ __forceinline__ int swizzle(int q) { return (q & 7) * 8; }
  // where in a stage warp i leaves column `col` of query q: in its own box of K, queries 8 to 15 in that of V
  static __device__ __forceinline__ int sum_at(int i, int q, int col) {
    return (q >> 3) * S::kTileBytes + i * S::kBoxBytes + ((q & 7) * D + (col ^ swizzle(q))) * 4;
  }
  static_assert(8 * D * 4 <= S::kBoxBytes, "eight queries' sums fit a box");
  __device__ __forceinline__ float sum(int u, int nd, int e) const {  // column 8 nd + 2 t + e of query g + 8 u
    return kRowsOf == 2 ? o[nd][2 * u + e] : o[nd][e] + o[nd][2 + e];
  }
  __device__ __forceinline__ void leave_sums(unsigned char* stage, int warp) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
    for (int u = 0; u < kRowsOf; ++u)
#pragma unroll
      for (int nd = 0; nd < D / 8; ++nd)
        *reinterpret_cast<float2*>(stage + sum_at(warp, g + 8 * u, nd * 8 + 2 * t)) = make_float2(sum(u, nd, 0), sum(u, nd, 1));
  }
  // the output of a head that is this warp's alone
  __device__ __forceinline__ void finish(const PageParams& p, size_t q_row, int queries) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
    for (int u = 0; u < kRowsOf; ++u) {
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 1);
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 2);
      if (g + 8 * u >= queries) continue;
      const size_t row = q_row + g + 8 * u;
#pragma unroll
      for (int nd = 0; nd < D / 8; ++nd)
        reinterpret_cast<uint32_t*>(p.out)[row * (D / 2) + nd * 4 + t] = pack_bf16(sum(u, nd, 0) / l[u], sum(u, nd, 1) / l[u]);
      if (p.lse && t == 0) p.lse[row] = (m[u] + fast_log2(l[u])) * kLn2;
    }
  }
};

// ---- fp32 ------------------------------------------------------------------------------------------
// A warp has kWarpRows rows of a tile: for the logits lane % kWarpRows is the row and the lanes that share it split
// its pieces; for the product with V a lane has D / 32 columns.
template <int D, int Q>
struct PlainWarp {
  using S = Shape<D, false, Q>;
  static constexpr int kRows = S::kWarpRows, kSplit = 32 / kRows, kPieces = D / 4 / kSplit, kCols = D / 32;
  static constexpr bool kOwnQueries = kRows == kBoxRows;  // a copy per warp (which may have its own head), or one
  const float* qs;        // [Q][D] in shared memory
  float m[Q], l[Q], o[Q][kCols];

  __device__ __forceinline__ void begin(const PageParams& p, size_t q_row, int queries, float* q_mem) {
    // (all warps are through with the queries before: they have met)
    if (kOwnQueries) __syncwarp();
    for (int i = kOwnQueries ? threadIdx.x & 31 : threadIdx.x; i < Q * (D / 4); i += kOwnQueries ? 32 : kConsumers * 32)
      reinterpret_cast<float4*>(q_mem)[i] = i / (D / 4) < queries
          ? reinterpret_cast<const float4*>(p.q)[q_row * (D / 4) + i] : make_float4(0.f, 0.f, 0.f, 0.f);
    if (kOwnQueries) __syncwarp();
    else meet();
    qs = q_mem;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      m[q] = -INFINITY;
      l[q] = 0.f;
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[q][c] = 0.f;
    }
  }

  template <class Wait>
  __device__ __forceinline__ bool tile(uint32_t k_tile, uint32_t v_tile, int r0, int valid, const Logit& logit,
                                       float* probs, Wait v_ready) {
    const int lane = threadIdx.x & 31, row = lane % kRows, share = lane / kRows;
    float z[Q] = {};
#pragma unroll 4
    for (int i = 0; i < kPieces; ++i) {
      const int c = i * kSplit + share;  // (neighbouring pieces: no bank conflicts among the queries')
      float4 k;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(k.x), "=f"(k.y), "=f"(k.z), "=f"(k.w)
                   : "r"(piece_at<S>(k_tile, r0 + row, c)));
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const float4 a = *reinterpret_cast<const float4*>(qs + q * D + 4 * c);
        z[q] = fmaf(a.x, k.x, fmaf(a.y, k.y, fmaf(a.z, k.z, fmaf(a.w, k.w, z[q]))));
      }
    }
    float corr[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
      for (int w = kRows; w < 32; w *= 2) z[q] += __shfl_xor_sync(0xffffffffu, z[q], w);
      z[q] = row < valid ? logit.of(z[q]) : -INFINITY;
      float best = z[q];
#pragma unroll
      for (int w = 1; w < kRows; w *= 2) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, w));
      const float m_new = fmaxf(m[q], best), ref = finite_ref(m_new);
      corr[q] = fast_exp2(m[q] - ref);
      m[q] = m_new;
      z[q] = fast_exp2(z[q] - ref);
      l[q] = l[q] * corr[q] + (share == 0 ? z[q] : 0.f);  // a lane's own rows
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[q][c] *= corr[q];
    }
    __syncwarp();  // (the probabilities of the tile before have been read)
    if (share == 0)
#pragma unroll
      for (int q = 0; q < Q; q += 4)
        *reinterpret_cast<float4*>(probs + row * Q + q) = make_float4(z[q], z[q + 1], z[q + 2], z[q + 3]);
    __syncwarp();
    if (!v_ready()) return false;
#pragma unroll 4
    for (int r = 0; r < kRows; ++r) {
      if (r >= valid) break;  // rows behind the last one may hold anything
      float v[kCols];
      if constexpr (kCols == 4)
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
                     : "r"(piece_at<S>(v_tile, r0 + r, lane)));
      else
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1])
                     : "r"(piece_at<S>(v_tile, r0 + r, lane / 2) + (lane & 1) * 8));
#pragma unroll
      for (int q = 0; q < Q; q += 4) {
        const float4 pr = *reinterpret_cast<const float4*>(probs + r * Q + q);
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          o[q][c] = fmaf(pr.x, v[c], o[q][c]);
          o[q + 1][c] = fmaf(pr.y, v[c], o[q + 1][c]);
          o[q + 2][c] = fmaf(pr.z, v[c], o[q + 2][c]);
          o[q + 3][c] = fmaf(pr.w, v[c], o[q + 3][c]);
        }
      }
    }
    return true;
  }

  __device__ __forceinline__ void leave_stats(float2* ml) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) l[q] += __shfl_xor_sync(0xffffffffu, l[q], w);
      if ((threadIdx.x & 31) == 0) ml[q] = make_float2(m[q], l[q]);
    }
  }
  // where in a stage warp i leaves four columns from `col` on of query q: in its own box of K; or, where a box is two
  // warps', in the q-th of its own rows
  static __device__ __forceinline__ int sum_at(int i, int q, int col) {
    return kRows == kBoxRows ? i * S::kBoxBytes + (q * D + col) * 4 : (int)piece_at<S>(0u, i * kRows + q, col / 4);
  }
  static_assert(Q * D * 4 <= kRows * S::kRowBytes, "the queries' sums fit a warp's rows");
  __device__ __forceinline__ void leave_sums(unsigned char* stage, int warp) {
    const int col = (threadIdx.x & 31) * kCols;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      float* to = reinterpret_cast<float*>(stage + sum_at(warp, q, col & ~3)) + (col & 3);
#pragma unroll
      for (int j = 0; j < kCols; ++j) to[j] = o[q][j];
    }
  }
  __device__ __forceinline__ void finish(const PageParams& p, size_t q_row, int queries) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) l[q] += __shfl_xor_sync(0xffffffffu, l[q], w);
      if (q >= queries) continue;
      float* to = reinterpret_cast<float*>(p.out) + (q_row + q) * D + lane * kCols;
#pragma unroll
      for (int j = 0; j < kCols; ++j) to[j] = o[q][j] / l[q];
      if (p.lse && lane == 0) p.lse[q_row + q] = (m[q] + fast_log2(l[q])) * kLn2;
    }
  }
};

template <bool BF16>
__device__ __forceinline__ void store4(void* out, size_t at, float4 x) {  // `at`: first of four elements
  if constexpr (BF16)
    *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(out) + at) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
  else
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(out) + at) = x;
}

// The partial results of `n` parts of a head, from CTA `w0` on (there the last of its part, then the first ones),
// joined in order: a warp per query.
template <int D, bool BF16, int Q>
__device__ __forceinline__ void join_parts(const PageParams& p, int w0, int n, int queries, size_t q_row) {
  constexpr int kCols = D / 32, kAhead = 8;
  using Cols = typename std::conditional<D == 128, float4, float2>::type;
  const int lane = threadIdx.x & 31;
  auto slot = [&](int i) { return (size_t)(w0 + i) * 2 + (i == 0); };
  for (int q = threadIdx.x >> 5; q < queries; q += kConsumers) {
    float top = -INFINITY;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, __ldcg(p.part_ml + slot(i) * Q + q).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float ref = finite_ref(top);
    float acc[kCols] = {}, l = 0.f;
    for (int s0 = 0; s0 < n; s0 += 32) {
      const float2 ml = s0 + lane < n ? __ldcg(p.part_ml + slot(s0 + lane) * Q + q) : make_float2(-INFINITY, 0.f);
      const float w = fast_exp2(ml.x - ref);
      const int end = min(32, n - s0);
      for (int i0 = 0; i0 < end; i0 += kAhead) {
        Cols v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          if (i0 + j < end) v[j] = __ldcg(reinterpret_cast<const Cols*>(p.part + (slot(s0 + i0 + j) * Q + q) * D) + lane);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          if (i0 + j >= end) break;
          const float wi = __shfl_sync(0xffffffffu, w, i0 + j);
          const float* f = reinterpret_cast<const float*>(&v[j]);
#pragma unroll
          for (int c = 0; c < kCols; ++c) acc[c] = fmaf(wi, f[c], acc[c]);
          l = fmaf(wi, __shfl_sync(0xffffffffu, ml.y, i0 + j), l);
        }
      }
    }
    const size_t at = (q_row + q) * D + lane * kCols;
    if constexpr (D == 128) {
      store4<BF16>(p.out, at, make_float4(acc[0] / l, acc[1] / l, acc[2] / l, acc[3] / l));
    } else if constexpr (BF16) {
      *reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at) = pack_bf16(acc[0] / l, acc[1] / l);
    } else {
      *reinterpret_cast<float2*>(reinterpret_cast<float*>(p.out) + at) = make_float2(acc[0] / l, acc[1] / l);
    }
    if (p.lse && lane == 0) p.lse[q_row + q] = (top + fast_log2(l)) * kLn2;
  }
}

// How the line of tiles is cut (the same in every CTA: it follows from the row counts).
struct Plan {
  long long total;   // tiles of all portions
  int parts;         // CTAs that have a part
  int piece;         // > 0: a portion's tiles in pieces of at most so many, one per CTA; 0: equal parts of the line
  int by_warp;       // 1: whole heads per warp
};

// Heads that are short against a warp's share go whole to warps, which then need not meet.  Else, where few CTAs have
// work, a portion is cut into pieces of 128 or 256 KB, no more than there are CTAs; and where there is more, the line
// into equal parts.
template <class S>
__device__ __forceinline__ Plan plan_of(const PageParams& p, const Counts& all) {
  Plan plan = {(long long)all.tiles * p.subs, 0, 0, 0};
  const long long grid = gridDim.x;
  if (S::kWarpRows == kBoxRows && p.subs == 1 && 2 * all.most * grid * kConsumers <= all.boxes) {
    plan.by_warp = 1;
    plan.parts = (int)grid;
  } else if ((long long)all.small * p.subs <= grid) {
    plan.piece = S::kSmall;
    plan.parts = all.small * p.subs;
  } else if ((long long)all.large * p.subs <= grid) {
    plan.piece = S::kLarge;
    plan.parts = all.large * p.subs;
  } else {
    plan.parts = (int)min(grid, plan.total);
  }
  return plan;
}

// What a CTA leaves of a portion that others have parts of.
struct Pending {
  int w0, n, queries;  // parts w0 ... w0 + n - 1; n = 0: nothing
  size_t q_row;
};

template <int D, bool BF16, int Q>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
decode_pages_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ PageParams p) {
  using S = Shape<D, BF16, Q>;
  using Warp = typename std::conditional<BF16, TensorWarp<D, Q>, PlainWarp<D, Q>>::type;
  constexpr int kWarpsAll = kThreads / 32;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t full_k[S::kStages], full_v[S::kStages], empty[S::kStages];
  __shared__ Ctl ctl;
  __shared__ int issued, last_one[2];
  __shared__ Start start;
  __shared__ int cuts[kConsumers + 1], cut_at[kConsumers + 1];  // by warp: their first heads, and boxes before those
  __shared__ Counts sums[kWarpsAll];
  __shared__ float2 stats[kConsumers][Q];
  __shared__ __align__(16) float q_mem[BF16 ? 4 : (Warp::kOwnQueries ? kConsumers : 1) * Q * D];  // fp32: the queries
  __shared__ __align__(16) float prob_mem[BF16 ? 4 : kConsumers * S::kWarpRows * Q];
  const Cache& c = p.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;

  if (tid == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(smem_u32(&full_k[s]), 1);
      mbar_init(smem_u32(&full_v[s]), 1);
      mbar_init(smem_u32(&empty[s]), kConsumers);
    }
    ctl.abort_flag = 0;
    ctl.wait_cycles = p.wait_cycles;
    issued = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  in_stream_order();

  // ---- the cut, and this CTA's part -----------------------------------------------------------------
  Plan plan;
  long long at0 = 0, at1 = 0;
  {
    const int share = (p.heads + kThreads - 1) / kThreads;
    const int h0 = min(p.heads, tid * share), h1 = min(p.heads, h0 + share);
    Counts mine = {};
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
      const int len = head_len(p, h);
      const int tiles = tiles_of<S>(len), boxes = (len + kBoxRows - 1) / kBoxRows;
      mine.add({tiles, boxes, (tiles + S::kSmall - 1) / S::kSmall, (tiles + S::kLarge - 1) / S::kLarge, boxes});
      if (len == 0 && h % (int)gridDim.x == (int)blockIdx.x) {  // no rows: zeros
        const int prob = h / c.n_kv_heads, kvh = h - prob * c.n_kv_heads;
        const size_t row = (size_t)prob * c.n_q_heads + (size_t)kvh * c.group;
        for (int i = 0; i < c.group * D; i += 4) store4<BF16>(p.out, row * D + i, make_float4(0.f, 0.f, 0.f, 0.f));
        if (p.lse)
          for (int i = 0; i < c.group; ++i) p.lse[row + i] = -INFINITY;
      }
    }
    const Counts of_warp = {__reduce_add_sync(0xffffffffu, mine.tiles), __reduce_add_sync(0xffffffffu, mine.boxes),
                            __reduce_add_sync(0xffffffffu, mine.small), __reduce_add_sync(0xffffffffu, mine.large),
                            __reduce_max_sync(0xffffffffu, mine.most)};
    if (lane == 0) sums[warp] = of_warp;
    __syncthreads();
    Counts all = {}, warps_before = {};
    for (int w = 0; w < kWarpsAll; ++w) {
      if (w == warp) warps_before = all;
      all.add(sums[w]);
    }
    plan = plan_of<S>(p, all);
    if ((int)blockIdx.x >= plan.parts) return;
    // what the cut counts, up to this thread's heads and in them
    const auto counted = [&](const Counts& x) {
      return plan.by_warp ? x.boxes : plan.piece == S::kSmall ? x.small : plan.piece ? x.large : x.tiles;
    };
    const int here = counted(mine);
    int incl = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const int before = counted(warps_before) + incl - here;
    if (plan.by_warp) {
      const long long workers = (long long)gridDim.x * kConsumers;
      for (int k = 0; k <= kConsumers; ++k) {  // the first head whose boxes begin at the cut or behind it
        const int cut = (int)(all.boxes * ((long long)blockIdx.x * kConsumers + k) / workers);
        if (cut == 0 && tid == 0) cuts[k] = cut_at[k] = 0;
        if (before < cut && cut <= before + here) {
          int at = before, h = h0;
          for (; at < cut; ++h) at += (head_len(p, h) + kBoxRows - 1) / kBoxRows;
          cuts[k] = h;
          cut_at[k] = at;
        }
      }
    } else {
      // the unit of the line, a tile or a piece, that this CTA's part begins with
      at0 = plan.piece ? (long long)blockIdx.x : plan.total * blockIdx.x / plan.parts;
      at1 = plan.total * (blockIdx.x + 1ll) / plan.parts;
      const long long first = (long long)before * p.subs;
      if (at0 >= first && at0 < first + (long long)here * p.subs) {
        const int size = plan.piece ? plan.piece : 1;
        const auto units = [&](int h) { return (tiles_of<S>(head_len(p, h)) + size - 1) / size; };
        long long at = first;
        int h = h0, n = units(h);
        while (at + (long long)n * p.subs <= at0) {
          at += (long long)n * p.subs;
          n = units(++h);
        }
        const int sub = (int)((at0 - at) / n), i = (int)((at0 - at) % n);
        const long long tiles = tiles_of<S>(head_len(p, h));
        if (plan.piece)
          start = {h, sub, (int)(tiles * i / n), (int)(tiles * (i + 1) / n), (int)at0 - i, n};
        else
          start = {h, sub, i, 0, 0, 0};
      }
    }
    __syncthreads();
  }
  int stage = 0, use = 0;
  bool alive = true;
  const auto wait = [&](uint64_t* bar, int parity) {  // the same in all lanes
    return __all_sync(0xffffffffu, wait_bar(smem_u32(bar), parity, &ctl, p.status)) != 0;
  };
  const auto next_stage = [&] {
    if (++stage == S::kStages) {
      stage = 0;
      ++use;
    }
  };
  // first row of the pool that a box of rows `row` ... is in (a page that is none of the pool: behind the pool's
  // rows, where copies give zeros)
  const auto place = [&](int h, int row) {
    const int page = p.table[(size_t)(p.first_head + h) * c.max_pages + (row >> c.page_shift)];
    return (unsigned)page < (unsigned)c.n_pages ? (page << c.page_shift) + (row & (c.page_rows - 1))
                                                : c.n_pages << c.page_shift;
  };

  if (plan.by_warp) {
    if constexpr (S::kWarpRows == kBoxRows) {
      int stages = 0;  // as many as the warp with most boxes has
#pragma unroll
      for (int k = 0; k < kConsumers; ++k) stages = max(stages, cut_at[k + 1] - cut_at[k]);
      if (warp == kConsumers) {
        // ---- producer: lanes 2 i and 2 i + 1 walk the heads of warp i, for K and for V; box i of a stage is warp i's
        const int of = min(lane >> 1, kConsumers - 1);
        const bool v = lane & 1, walks = lane < 2 * kConsumers;
        int h = cuts[of], end = walks ? cuts[of + 1] : 0, row = 0, len = 0;
        const auto advance = [&] {  // to the next row that begins a box, in a head that has rows
          while (h < end && row >= len) {
            if (len > 0) ++h;
            len = h < end ? head_len(p, h) : 0;
            row = 0;
            if (len == 0 && h < end) ++h;
          }
        };
        advance();
        int at = h < end ? place(h, row) : 0;
        for (; stages > 0; --stages) {
          if (use > 0 && !(alive = wait(&empty[stage], (use - 1) & 1))) break;
          const int boxes = __popc(__ballot_sync(0xffffffffu, h < end)) / 2;
          if (lane == 0) {
            mbar_expect_tx(smem_u32(&full_k[stage]), boxes * S::kBoxBytes);
            mbar_expect_tx(smem_u32(&full_v[stage]), boxes * S::kBoxBytes);
            ++issued;
          }
          __syncwarp();
          if (h < end) {
            tma_load_3d(ring + stage * S::kStageBytes + (v ? S::kTileBytes : 0) + of * S::kBoxBytes, v ? &map_v : &map_k, 0,
                        at, 0, smem_u32(v ? &full_v[stage] : &full_k[stage]));
            row += kBoxRows;
            advance();
            if (h < end) at = place(h, row);
          }
          next_stage();
          __syncwarp();
        }
      } else {
        // ---- consumers: their own heads
        Warp w;
        const Logit logit(c);
        float* const probs = prob_mem + (BF16 ? 0 : warp * S::kWarpRows * Q);
        for (int h = cuts[warp]; h < cuts[warp + 1] && alive; ++h) {
          const int len = head_len(p, h);
          if (len == 0) continue;
          const int prob = h / c.n_kv_heads, kvh = h - prob * c.n_kv_heads;
          const size_t q_row = (size_t)prob * c.n_q_heads + (size_t)kvh * c.group;
          if constexpr (BF16) w.begin(p, q_row, c.group);
          else w.begin(p, q_row, c.group, q_mem + warp * Q * D);
          for (int row = 0; row < len; row += kBoxRows) {
            const uint32_t k_tile = ring + stage * S::kStageBytes;
            if (!(alive = wait(&full_k[stage], use & 1))) break;
            alive = w.tile(k_tile, k_tile + S::kTileBytes, warp * kBoxRows, min(kBoxRows, len - row), logit, probs,
                           [&] { return wait(&full_v[stage], use & 1); });
            if (!alive) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
            next_stage();
            --stages;
          }
          if (alive) w.finish(p, q_row, c.group);
        }
        for (; stages > 0 && alive; --stages) {  // with boxes of other warps only
          alive = wait(&full_k[stage], use & 1);
          if (alive && lane == 0) mbar_arrive(smem_u32(&empty[stage]));
          next_stage();
        }
      }
    }
  } else if (warp == kConsumers) {
    // ---- producer ----------------------------------------------------------------------------------
    long long left = plan.piece ? start.end - start.tile : at1 - at0;
    int sub = start.sub, t0 = start.tile;  // of the head in hand; 0 in the heads that follow
    for (int h = start.head; left > 0 && alive; ++h, sub = 0) {
      const int len = head_len(p, h), n = tiles_of<S>(len);
      if (n == 0) continue;
      for (; sub < p.subs && left > 0 && alive; ++sub, t0 = 0) {
        const int t1 = (int)min((long long)n, t0 + left);
        left -= t1 - t0;
        for (int t = t0; t < t1; ++t) {
          const int row0 = t * S::kTile;
          const int boxes = min(S::kTile / kBoxRows, (len - row0 + kBoxRows - 1) / kBoxRows);
          // lane 2 i + v: box i of K or V
          const int at = lane < 2 * boxes ? place(h, row0 + (lane >> 1) * kBoxRows) : 0;
          if (use > 0 && !(alive = wait(&empty[stage], (use - 1) & 1))) break;
          if (lane == 0) {
            mbar_expect_tx(smem_u32(&full_k[stage]), boxes * S::kBoxBytes);
            mbar_expect_tx(smem_u32(&full_v[stage]), boxes * S::kBoxBytes);
            ++issued;
          }
          __syncwarp();
          if (lane < 2 * boxes) {
            const bool v = lane & 1;
            tma_load_3d(ring + stage * S::kStageBytes + (v ? S::kTileBytes : 0) + (lane >> 1) * S::kBoxBytes,
                        v ? &map_v : &map_k, 0, at, 0, smem_u32(v ? &full_v[stage] : &full_k[stage]));
          }
          next_stage();
        }
      }
    }
  } else {
    // ---- consumers ---------------------------------------------------------------------------------
    Warp w;
    const Logit logit(c);
    float* const probs = prob_mem + (BF16 ? 0 : warp * S::kWarpRows * Q);
    Pending begun = {}, ended = {};  // the portion that the part begins in, and the one that it ends in
    long long left = plan.piece ? start.end - start.tile : at1 - at0;
    int sub = start.sub, t0 = start.tile;
    long long at = at0 - t0;  // first tile of the head's portion on the line
    for (int h = start.head; left > 0 && alive; ++h, sub = 0) {
      const int len = head_len(p, h), n = tiles_of<S>(len);
      if (n == 0) continue;
      const int prob = h / c.n_kv_heads, kvh = h - prob * c.n_kv_heads;
      for (; sub < p.subs && left > 0; ++sub, t0 = 0) {
        const int t1 = (int)min((long long)n, t0 + left);
        const int queries = min(p.per_sub, c.group - sub * p.per_sub);
        const size_t q_row = (size_t)prob * c.n_q_heads + (size_t)kvh * c.group + sub * p.per_sub;
        if constexpr (BF16) w.begin(p, q_row, queries);
        else w.begin(p, q_row, queries, q_mem + (Warp::kOwnQueries ? warp * Q * D : 0));
        for (int t = t0; t < t1; ++t) {
          const uint32_t k_tile = ring + stage * S::kStageBytes, v_tile = k_tile + S::kTileBytes;
          const int r0 = warp * S::kWarpRows, valid = min(S::kWarpRows, len - t * S::kTile - r0);
          if (!(alive = wait(&full_k[stage], use & 1))) break;
          const auto v_ready = [&] { return wait(&full_v[stage], use & 1); };
          alive = valid > 0 ? w.tile(k_tile, v_tile, r0, valid, logit, probs, v_ready) : v_ready();
          if (!alive) break;
          if (t + 1 < t1) {  // (the last stage is kept for the meeting)
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
            next_stage();
          }
        }
        // The warps meet: each leaves its maxima and sums, and what it has summed of V in the memory of its own rows
        // of the last stage, which no other warp reads.
        unsigned char* const last = smem_raw + (ring - smem_u32(smem_raw)) + stage * S::kStageBytes;
        w.leave_stats(stats[warp]);
        __syncwarp();
        w.leave_sums(last, warp);
        alive = meet_all(alive);
        if (!alive) break;
        const bool whole = t0 == 0 && t1 == n;
        const size_t slot = (size_t)blockIdx.x * 2 + (t0 == 0);
        for (int e = tid; e < queries * (D / 4); e += kConsumers * 32) {
          const int q = e / (D / 4), col = e % (D / 4) * 4;
          const float top = top_of<Q>(stats, q);
          float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
          float l = 0.f;
#pragma unroll
          for (int i = 0; i < kConsumers; ++i) {
            const float4 f = *reinterpret_cast<const float4*>(last + Warp::sum_at(i, q, col));
            const float s = fast_exp2(stats[i][q].x - finite_ref(top));
            a = make_float4(fmaf(f.x, s, a.x), fmaf(f.y, s, a.y), fmaf(f.z, s, a.z), fmaf(f.w, s, a.w));
            l = fmaf(stats[i][q].y, s, l);
          }
          if (whole) {
            store4<BF16>(p.out, (q_row + q) * D + col, make_float4(a.x / l, a.y / l, a.z / l, a.w / l));
            if (p.lse && col == 0) p.lse[q_row + q] = (top + fast_log2(l)) * kLn2;
          } else {
            *reinterpret_cast<float4*>(p.part + (slot * Q + q) * D + col) = a;
            if (col == 0) p.part_ml[slot * Q + q] = make_float2(top, l);
          }
        }
        fence_async_proxy();  // (the stage was written; the next copy into it comes after)
        meet();
        if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
        next_stage();
        if (!whole) {
          // the parts that the portion's tiles lie in
          Pending x = {start.first, start.pieces, queries, q_row};
          if (!plan.piece) {
            x.w0 = (int)(((at + 1) * plan.parts - 1) / plan.total);
            x.n = (int)(((at + n) * plan.parts - 1) / plan.total) + 1 - x.w0;
          }
          if (t0 == 0) ended = x;
          else begun = x;
        }
        left -= t1 - t0;
        at += n;
      }
    }
    // Portions that other CTAs have parts of, when this CTA is through: who comes last joins them.
    if (alive && (begun.n || ended.n)) {
      __threadfence();
      meet();
      if (tid == 0 && begun.n) last_one[0] = atomicAdd(p.counters + begun.w0, 1) == begun.n - 1;
      if (tid == 32 && ended.n) last_one[1] = atomicAdd(p.counters + ended.w0, 1) == ended.n - 1;
      meet();
      __threadfence();
      if (begun.n && last_one[0]) {
        join_parts<D, BF16, Q>(p, begun.w0, begun.n, begun.queries, begun.q_row);
        if (tid == 0) p.counters[begun.w0] = 0;
      }
      if (ended.n && last_one[1]) {
        join_parts<D, BF16, Q>(p, ended.w0, ended.n, ended.queries, ended.q_row);
        if (tid == 0) p.counters[ended.w0] = 0;
      }
    }
  }
  // after a wait that gave up: no CTA leaves under a copy of its own
  __syncthreads();
  if (ctl.abort_flag && tid == 0) {
    for (int i = max(0, issued - S::kStages); i < issued; ++i) {
      wait_bar(smem_u32(&full_k[i % S::kStages]), (i / S::kStages) & 1, &ctl, p.status, false);
      wait_bar(smem_u32(&full_v[i % S::kStages]), (i / S::kStages) & 1, &ctl, p.status, false);
    }
  }
}

// A group's queries in portions that a warp can hold.
struct Portions {
  int held, subs, per_sub;
};
Portions portions_of(const Cache& c) {
  const int most = c.dtype == LAVA_BF16 ? 16 : 8;
  const int subs = (c.group + most - 1) / most, per_sub = (c.group + subs - 1) / subs;
  return {per_sub <= most / 2 ? most / 2 : most, subs, per_sub};
}

constexpr size_t kStatusBytes = 256;
int most_ctas() { return kCtasPerSm * (sm_count() > 0 ? sm_count() : 148); }
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
size_t counter_bytes() { return up256(most_ctas() * sizeof(int)); }
size_t slots_of(const Cache& c) { return (size_t)most_ctas() * 2 * portions_of(c).held; }

template <int D, bool BF16, int Q>
lava_status launch(const CUtensorMap& map_k, const CUtensorMap& map_v, PageParams& p, cudaStream_t stream) {
  using S = Shape<D, BF16, Q>;
  const auto kernel = decode_pages_kernel<D, BF16, Q>;
  const lava_status rc = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem),
                                    "paged decode attention attribute");
  if (rc != LAVA_OK) return rc;
  const long long most = ((((long long)p.c.max_pages << p.c.page_shift) + S::kTile - 1) / S::kTile) * p.heads * p.subs;
  const int grid = (int)std::min<long long>(most_ctas(), most);
  const cudaError_t e = launch_in_order(kernel, grid, kThreads, S::kSmem, stream, map_k, map_v, p);
  count_launches(1);
  return check_cuda(e, "paged decode attention launch");
}

}  // namespace
}  // namespace lava

using namespace lava;

extern "C" {

size_t lava_cache_workspace_bytes(const lava_cache_desc* cache) {
  Cache c;
  if (make_cache(cache, &c) != LAVA_OK) return 0;
  return kStatusBytes + counter_bytes() + up256(slots_of(c) * c.head_dim * sizeof(float)) +
         up256(slots_of(c) * sizeof(float2));
}

lava_status lava_decode_attention_pages(const lava_cache_desc* cache, int32_t first_layer, int32_t n_layers,
                                        const void* q, const void* k_pages, const void* v_pages,
                                        const int32_t* page_table, const int32_t* head_rows, void* out, float* lse,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  PageParams p = {};
  lava_status rc = make_cache(cache, &p.c);
  if (rc != LAVA_OK) return rc;
  const Cache& c = p.c;
  if (n_layers < 1 || first_layer < 0 || first_layer > c.n_layers - n_layers)
    return fail(LAVA_ERR_INVALID_ARG, "layers %d ... %lld are not all in a cache of %d", first_layer,
                (long long)first_layer + n_layers - 1, c.n_layers);
  if (!q || !k_pages || !v_pages || !page_table || !head_rows || !out)
    return fail(LAVA_ERR_INVALID_ARG, "NULL argument");
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out))
    return fail(LAVA_ERR_INVALID_ARG, "q, k_pages, v_pages and out must be 16-byte aligned");
  if (((long long)n_layers * c.batch * c.n_kv_heads) >= (1ll << 35) / ((long long)c.max_pages << c.page_shift))
    return fail(LAVA_ERR_UNSUPPORTED, "the heads of the call times the rows of a head must stay below 2^35");
  const size_t need = lava_cache_workspace_bytes(cache);
  if (!workspace || workspace_bytes < need)
    return fail(LAVA_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
  if (!aligned16(workspace)) return fail(LAVA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  CUtensorMap map_k, map_v;
  rc = encode_pages_map(c, k_pages, &map_k);
  if (rc == LAVA_OK) rc = encode_pages_map(c, v_pages, &map_v);
  if (rc != LAVA_OK) return rc;
  const Portions portions = portions_of(c);
  p.first_head = first_layer * c.batch * c.n_kv_heads;
  p.heads = n_layers * c.batch * c.n_kv_heads;
  p.subs = portions.subs;
  p.per_sub = portions.per_sub;
  p.q = q;
  p.table = page_table;
  p.rows = head_rows;
  p.out = out;
  p.lse = lse;
  char* ws = (char*)workspace;
  p.status = (unsigned*)ws;
  p.counters = (int*)(ws + kStatusBytes);
  p.part = (float*)(ws + kStatusBytes + counter_bytes());
  p.part_ml = (float2*)((char*)p.part + up256(slots_of(c) * c.head_dim * sizeof(float)));
  p.wait_cycles = options().wait_limit_cycles;
  cudaStream_t st = (cudaStream_t)stream;
  if (c.dtype == LAVA_BF16) {
    if (c.head_dim == 128)
      return portions.held == 8 ? launch<128, true, 8>(map_k, map_v, p, st) : launch<128, true, 16>(map_k, map_v, p, st);
    return portions.held == 8 ? launch<64, true, 8>(map_k, map_v, p, st) : launch<64, true, 16>(map_k, map_v, p, st);
  }
  if (c.head_dim == 128)
    return portions.held == 4 ? launch<128, false, 4>(map_k, map_v, p, st) : launch<128, false, 8>(map_k, map_v, p, st);
  return portions.held == 4 ? launch<64, false, 4>(map_k, map_v, p, st) : launch<64, false, 8>(map_k, map_v, p, st);
}

}  // extern "C"
