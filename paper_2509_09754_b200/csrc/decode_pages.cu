// Attention of one new token over the pages of a paged cache.
//
//     x_i = scale * q . K[i]  (capped: c tanh(x / c)),   out = sum_i e^(x_i - m) V[i] / sum_i e^(x_i - m)
//
// One pass over the rows with a running maximum m and sum, logits in the base-2 domain.  All query heads of a KV
// head's group share the read of its rows.  What has to be read is the rows, once; everything else is small, so the
// kernel is built to keep copies in flight:
//
// The rows of all heads, in boxes of 16, form one line, which is cut into equal parts, one per CTA, two CTAs per SM: heads
// of any lengths load all SMs alike.  Rows are worked on in tiles (64 rows of a head; 32 of 512 bytes), and a tile is in
// the part that its first box is in.  Row counts live on the device, so every CTA finds its part
// itself.  A producer warp walks the part: it looks up the tile's pages and has TMA fetch K and V in boxes (16 rows are
// the least page) into a ring of stages; boxes behind a head's last row are not fetched.  Four warps consume a
// tile, a quarter of its rows each, with maxima and sums of their own until the head or the part ends; then they meet
// through the memory of the last stage.  A head inside one part is finished there.  Of a head that continues in other
// parts the partial result goes to memory; the CTA that comes last, as a counter tells, joins them in order.
//
// bf16: S = Q K^T and O += P V by mma.sync m16n8k16 (the tensor pipe is 18 % busy at the rate of HBM).  With up to 8
// queries the other 8 rows of the A operand are free: they carry what rounding the probabilities to bf16 left over, so
// the products with V keep 16 bits of every probability at no cost; with 9 to 16 queries a second product does.  More
// queries per KV head than 16 are taken 16 at a time.  fp32: lanes have a share of one or two rows for the logits, and
// some columns for the product with V; up to 8 queries at a time.
//
// Bound by HBM where the heads hold enough (64 x 8 heads of 2048 rows, bf16 of 128: 92 us, 5.8 TB/s where a copy has
// 6.6; 16 queries a head 106 us; fp32, 32 sequences: 88 us, with 8 queries a head 93), else by the chain of one CTA:
// counts, page table, rows, joining (5.5 us for short sequences, 8 to 10 where heads are split).
#include <algorithm>
#include <atomic>
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
  static constexpr int kPieceLog = kStageBytes == 32 * 1024 ? 1 : 2;  // of the tiles of the smallest pieces: 64 KB
  static_assert(kStageBytes << kPieceLog == 64 * 1024, "smallest pieces");
};

struct PageParams {
  Cache c;
  int first_head;          // of the call's first layer
  int heads;               // of the call's layers
  int subs, per_sub;       // a group's queries are taken in `subs` portions of `per_sub`
  int own_queries;         // a warp can have a head of its own
  int sms;
  const void* q;           // [layers, batch, H_q, d]
  const int* table;
  const int* rows;
  void* out;
  float* lse;
  float* part;             // [CTA][2][Q][D]: partial results of the part's first and last portion,
  float2* part_ml;         // [CTA][2][Q]: the maximum that they are relative to, and the sum
  int* counters;           // [CTA]: CTAs that have left their result of the portion that begins last in this one's part
  unsigned* status;
  long long wait_cycles;
  int sleep;               // waits sleep between two looks (0 where the limit is shorter than that)
};

struct Ctl {
  volatile int abort_flag;
  long long wait_cycles;
};

template <class S>
__device__ __forceinline__ int tiles_of(int len) {
  return (len + S::kTile - 1) / S::kTile;
}
__device__ __forceinline__ int boxes_of(int len) { return (len + kBoxRows - 1) / kBoxRows; }
// Sums over heads: boxes (the host has seen to it that they fit), and pieces of every size, each twice the one before, two
// in a word.  More pieces than a call has CTAs need not be told apart, so counts stop where 16 bits hold their sums.
constexpr int kSizes = 6, kMostPieces = 511;
struct Counts {
  int boxes;
  unsigned pieces[kSizes / 2];
  template <class S>
  static __device__ __forceinline__ Counts of(int len) {
    Counts x;
    x.boxes = boxes_of(len);
#pragma unroll
    for (int i = 0; i < kSizes; i += 2)
      x.pieces[i / 2] = min(pieces_of<S>(len, i), kMostPieces) | min(pieces_of<S>(len, i + 1), kMostPieces) << 16;
    return x;
  }
  template <class S>
  static __device__ __forceinline__ int pieces_of(int len, int size) {
    const int log = S::kPieceLog + size;
    return (tiles_of<S>(len) + (1 << log) - 1) >> log;
  }
  __device__ __forceinline__ Counts over_warp() const {
    Counts x;
    x.boxes = __reduce_add_sync(0xffffffffu, boxes);
#pragma unroll
    for (int i = 0; i < kSizes / 2; ++i) {
      const unsigned n = __reduce_add_sync(0xffffffffu, pieces[i]);
      x.pieces[i] = min(n & 0xffffu, 2u * kMostPieces) | min(n >> 16, 2u * kMostPieces) << 16;
    }
    return x;
  }
  __device__ __forceinline__ int of_size(int i) const { return pieces[i / 2] >> (i % 2 * 16) & 0xffffu; }
};
static_assert(32 * 2 * kMostPieces < 65536, "32 heads, or 32 segments");
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
    // (tanhf: around z = 1/4 capped logits are off by 2.4 * 2^-24 of themselves.  1 - 2 / (e^(2 z) + 1) with the fast
    // exponential cancels there, 6.8.  That / tanhf, us, 64 x 8 heads of 2048 rows, bf16: 91.6 / 92.4; with 16 queries a
    // head 115.7 / 118.1; of 64 columns 61.8 / 63.7.)
    return cap * tanhf(s * in);
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

// Rows behind a head's last one may hold anything: their probabilities are 0, so must they be.  By one warp.
template <class S>
__device__ __forceinline__ void clear_rows(uint32_t tile, int begin, int end) {
  constexpr int kPieces = S::kRowBytes / 16;
  for (int i = threadIdx.x & 31; i < (end - begin) * kPieces; i += 32)
    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(piece_at<S>(tile, begin + i / kPieces, i % kPieces)), "r"(0)
                 : "memory");
  fence_async_proxy();  // (before the next copy into this stage)
  __syncwarp();
}

// ---- bf16: tensor cores ----------------------------------------------------------------------------
// Thread (g = lane / 4, t = lane % 4) has query row g, and with 16 queries g + 8 too.
template <int D, int Q>
struct TensorWarp {
  using S = Shape<D, true, Q>;
  static constexpr int kRowsOf = Q / 8;
  // The queries lie in shared memory as the A operand's fragments, 16 bytes per lane: a copy per warp, which may have a
  // head of its own, or one (16 queries of 128 leave no room for four).  The next head's are on their way in registers.
  static constexpr int kFrags = D / 16 * 2 * kRowsOf / 4;
  static constexpr bool kOwnQueries = Q * D <= 1024;
  static constexpr int kNext = kOwnQueries ? kFrags : kFrags / kConsumers;
  static constexpr int kQueryBytes = kFrags * 512;  // of a copy
  uint4 next[kNext];
  float m[kRowsOf], l[kRowsOf], o[D / 8][4];

  __device__ __forceinline__ void fetch(const PageParams& p, size_t q_row, int queries) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3, first = kOwnQueries ? 0 : (threadIdx.x >> 5) * kNext;
    const uint32_t* qh = reinterpret_cast<const uint32_t*>(p.q) + (q_row + g) * (D / 2) + t;
#pragma unroll
    for (int j = 0; j < kNext; ++j) {
      const int i = first + j;  // k-steps 2 i and 2 i + 1 of rows g, or k-step i of rows g and g + 8
      const uint32_t* lo = qh + (kRowsOf == 1 ? 16 : 8) * i;
      const uint32_t* hi = kRowsOf == 1 ? lo + 8 : lo + 8 * (D / 2);
      const bool there = g < queries, other = kRowsOf == 1 ? there : g + 8 < queries;
      next[j] = kRowsOf == 1 ? make_uint4(there ? lo[0] : 0u, there ? lo[4] : 0u, there ? hi[0] : 0u, there ? hi[4] : 0u)
                             : make_uint4(there ? lo[0] : 0u, other ? hi[0] : 0u, there ? lo[4] : 0u, other ? hi[4] : 0u);
    }
  }

  // a head begins, whose queries have been fetched
  __device__ __forceinline__ void begin(unsigned char* q_mem) {
    const int lane = threadIdx.x & 31, first = kOwnQueries ? 0 : (threadIdx.x >> 5) * kNext;
    __syncwarp();  // (in a shared copy: all warps are through with the queries before, they have met)
#pragma unroll
    for (int j = 0; j < kNext; ++j) reinterpret_cast<uint4*>(q_mem)[(first + j) * 32 + lane] = next[j];
    if (kOwnQueries) __syncwarp();
    else meet();
#pragma unroll
    for (int u = 0; u < kRowsOf; ++u) {
      m[u] = -INFINITY;
      l[u] = 0.f;
    }
#pragma unroll
    for (int nd = 0; nd < D / 8; ++nd) o[nd][0] = o[nd][1] = o[nd][2] = o[nd][3] = 0.f;
  }

  // rows r0 ... r0 + 15 of the tile, of which `valid` (> 0) are there
  __device__ __forceinline__ void tile(uint32_t k_tile, uint32_t v_tile, int r0, int valid, const Logit& logit,
                                       const unsigned char* q_mem, float*) {
    const int lane = threadIdx.x & 31, t = lane & 3, mi = lane >> 3, r8 = lane & 7;
    float s[2][4] = {}, s2[2][4] = {};  // odd k-steps have sums of their own: shorter chains
    uint4 qa = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {  // matrices (keys 0-7, piece 2 ks), (0-7, 2 ks + 1), (8-15, ...)
      uint32_t b0, b1, b2, b3;
      ldmatrix_x4(b0, b1, b2, b3, piece_at<S>(k_tile, r0 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1)));
      if (kRowsOf == 2 || ks % 2 == 0)
        qa = reinterpret_cast<const uint4*>(q_mem)[(kRowsOf == 2 ? ks : ks / 2) * 32 + lane];
      const uint32_t a0 = kRowsOf == 2 || ks % 2 == 0 ? qa.x : qa.z, a1 = kRowsOf == 2 ? qa.y : 0u;
      const uint32_t a2 = kRowsOf == 2 ? qa.z : ks % 2 == 0 ? qa.y : qa.w, a3 = kRowsOf == 2 ? qa.w : 0u;
      float (&to)[2][4] = ks % 2 ? s2 : s;
      mma_bf16_16816(to[0][0], to[0][1], to[0][2], to[0][3], a0, a1, a2, a3, b0, b1);
      mma_bf16_16816(to[1][0], to[1][1], to[1][2], to[1][3], a0, a1, a2, a3, b2, b3);
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
          x[n][e] = 8 * n + 2 * t + e < valid ? logit.of(s[n][2 * u + e] + s2[n][2 * u + e]) : -INFINITY;
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
    if (valid < 16) clear_rows<S>(v_tile, r0 + valid, r0 + 16);
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
      const float inv = 1.f / l[u];
#pragma unroll
      for (int nd = 0; nd < D / 8; ++nd)
        reinterpret_cast<uint32_t*>(p.out)[row * (D / 2) + nd * 4 + t] = pack_bf16(sum(u, nd, 0) * inv, sum(u, nd, 1) * inv);
      if (p.lse && t == 0) p.lse[row] = (m[u] + fast_log2(l[u])) * kLn2;
    }
  }
};

// ---- fp32 ------------------------------------------------------------------------------------------
// A warp has kWarpRows rows of a tile.  For the logits a lane has kPer of them, lane % kLanes and on, and the lanes that
// have the same rows split their pieces; two rows, and half as many loads of the queries, wherever there are queries
// enough for the lanes to split.  For the product with V a lane has D / 32 columns.
template <int D, int Q>
struct PlainWarp {
  using S = Shape<D, false, Q>;
  static constexpr int kRows = S::kWarpRows, kPer = Q * kRows >= 64 ? 2 : 1, kLanes = kRows / kPer;
  static constexpr int kSplit = 32 / kLanes, kPieces = D / 4 / kSplit, kCols = D / 32;
  static constexpr bool kOwnQueries = kRows == kBoxRows;  // a copy per warp (which may have its own head), or one
  static constexpr int kQueryBytes = Q * D * 4;
  static constexpr int kNext = Q * D / 4 / (kOwnQueries ? 32 : 32 * kConsumers);
  static_assert(kNext >= 1, "a lane has a piece of the queries");
  // The lanes that share rows split the queries when the logits are summed: each has kOwn of them, from own0() on.
  static constexpr int kOwn = Q / kSplit;
  static_assert((kOwn == 1 || kOwn == 2) && kOwn * kSplit == Q, "queries of a lane");
  uint4 next[kNext];      // of the queries of the next head
  float m[kOwn], l[kOwn], o[Q][kCols];
  static __device__ __forceinline__ int own0() { return (threadIdx.x & 31) / kLanes * kOwn; }
  // query q's value among those that the lanes have of their own (the same for all rows)
  static __device__ __forceinline__ float of_query(const float (&x)[kOwn], int q) {
    return __shfl_sync(0xffffffffu, x[q % kOwn], q / kOwn * kLanes);
  }

  __device__ __forceinline__ void fetch(const PageParams& p, size_t q_row, int queries) {
    const int first = kOwnQueries ? threadIdx.x & 31 : threadIdx.x;
#pragma unroll
    for (int j = 0; j < kNext; ++j) {
      const int i = first + j * (kOwnQueries ? 32 : 32 * kConsumers);
      next[j] = i / (D / 4) < queries ? reinterpret_cast<const uint4*>(p.q)[q_row * (D / 4) + i] : uint4{};
    }
  }

  __device__ __forceinline__ void begin(unsigned char* q_mem) {
    const int first = kOwnQueries ? threadIdx.x & 31 : threadIdx.x;
    __syncwarp();  // (in a shared copy: all warps are through with the queries before, they have met)
#pragma unroll
    for (int j = 0; j < kNext; ++j)
      reinterpret_cast<uint4*>(q_mem)[first + j * (kOwnQueries ? 32 : 32 * kConsumers)] = next[j];
    if (kOwnQueries) __syncwarp();
    else meet();
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[q][c] = 0.f;
  }

  __device__ __forceinline__ void tile(uint32_t k_tile, uint32_t v_tile, int r0, int valid, const Logit& logit,
                                       const unsigned char* q_mem, float* probs) {
    const int lane = threadIdx.x & 31, row = lane % kLanes, share = lane / kLanes;
    const float* qs = reinterpret_cast<const float*>(q_mem);  // [Q][D]
    // the share's first piece: those of all shares neighbours, and no bank conflicts among eight lanes' pieces of K
    const int c0 = kLanes == 4 ? (share & 1) * 4 + share / 2 : share;
    float z[kPer][Q] = {};
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int c = i * kSplit + c0;
      float4 k[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(k[j].x), "=f"(k[j].y), "=f"(k[j].z), "=f"(k[j].w)
                     : "r"(piece_at<S>(k_tile, r0 + row + j * kLanes, c)));
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const float4 a = *reinterpret_cast<const float4*>(qs + q * D + 4 * c);
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          z[j][q] = fmaf(a.x, k[j].x, fmaf(a.y, k[j].y, fmaf(a.z, k[j].z, fmaf(a.w, k[j].w, z[j][q]))));
      }
    }
    // sums over the lanes that share rows, which halve their queries at every step
    int left = Q;
#pragma unroll
    for (int w = 16; w >= kLanes; w /= 2) {
      left /= 2;
      const bool upper = lane & w;
#pragma unroll
      for (int j = 0; j < kPer; ++j)
#pragma unroll
        for (int i = 0; i < Q / 2; ++i)
          if (i < left) {
            const float away = upper ? z[j][i] : z[j][left + i], mine = upper ? z[j][left + i] : z[j][i];
            z[j][i] = mine + __shfl_xor_sync(0xffffffffu, away, w);
          }
    }
    float corr[kOwn];
    bool moved = false;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      float best = -INFINITY;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        z[j][i] = row + j * kLanes < valid ? logit.of(z[j][i]) : -INFINITY;
        best = fmaxf(best, z[j][i]);
      }
#pragma unroll
      for (int w = 1; w < kLanes; w *= 2) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, w));
      const float m_new = fmaxf(m[i], best), ref = finite_ref(m_new);
      corr[i] = fast_exp2(m[i] - ref);
      moved |= m_new != m[i];
      m[i] = m_new;
      l[i] *= corr[i];
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        z[j][i] = fast_exp2(z[j][i] - ref);
        l[i] += z[j][i];  // a lane's own rows
      }
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const float x = of_query(corr, q);
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[q][c] *= x;
      }
    }
    __syncwarp();  // (the probabilities of the tile before have been read)
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      float* const to = probs + (row + j * kLanes) * Q + own0();
      if constexpr (kOwn == 2) *reinterpret_cast<float2*>(to) = make_float2(z[j][0], z[j][1]);
      else to[0] = z[j][0];
    }
    __syncwarp();
    if (valid < kRows) clear_rows<S>(v_tile, r0 + valid, r0 + kRows);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
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
  }

  // sums of the lanes' rows
  __device__ __forceinline__ void sum_rows() {
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
#pragma unroll
      for (int w = 1; w < kLanes; w *= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
  }
  __device__ __forceinline__ void leave_stats(float2* ml) {
    sum_rows();
    if ((threadIdx.x & 31) % kLanes == 0)
#pragma unroll
      for (int i = 0; i < kOwn; ++i) ml[own0() + i] = make_float2(m[i], l[i]);
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
    sum_rows();
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const float top = of_query(m, q), sum = of_query(l, q);
      if (q >= queries) continue;
      float* to = reinterpret_cast<float*>(p.out) + (q_row + q) * D + lane * kCols;
#pragma unroll
      for (int j = 0; j < kCols; ++j) to[j] = o[q][j] / sum;
      if (p.lse && lane == 0) p.lse[q_row + q] = (top + fast_log2(sum)) * kLn2;
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

template <class S>
constexpr int kBoxesOf = S::kTile / kBoxRows;  // boxes of a tile
constexpr int kPieceHeads = 1024;              // heads above which pieces are not counted

// How the line is cut (the same in every CTA: it follows from the row counts).
struct Plan {
  int by_warp;  // 1: whole heads per warp
  int piece;    // i > 0: a portion in pieces of size i - 1, one per CTA
  int parts;    // CTAs that have a part
  int total;    // boxes of all portions (the host has seen to it that 32 bits hold them)
};

// Heads that are short against a warp's share go whole to warps, which then need not meet.  Else, where there are CTAs
// for it, every CTA gets a piece of one portion: the whole of it where none is longer than 192 KB, else the smallest
// size that there are CTAs for (for 64 KB: SMs), up to 256 KB or 5/2 of an equal part.  Else the line is cut into equal
// parts.  These load the SMs better, but most of them end in two heads: two meetings, two partial results.
// Pieces / parts, us: 28 x 4 heads of 1024 rows 19.4 (of 256 KB) / 25.0, of 2000 27.8 (512 KB) / 32.6; 8 heads of 30000
// rows 29.5 (512 KB) / 33.6, of 60000 47.8 (1 MB) / 49.6; 128 heads of 2400 34.2 (1 MB) / 35.0, 256 of 200 12.3 (256 KB)
// / 14.9.  64 KB / 128: 8 heads of 600 rows 7.6 / 8.7, 64 of 150 8.1 / 8.9.  Whole / pieces: 64 of 80 rows, the longest
// of 300, 7.3 / 7.9; with heads of up to 256 KB whole 8.6 / 7.8.
// (SMs do not get equal shares of the bandwidth: of 64 x 8 heads of 2048 rows the first CTA is through
// after 68 us, the last after 86.  An eighth of the line in small parts for whoever is through did not pay: 105 us against
// 96, with a twelfth in fewer parts 101; every small part has its own meeting, partial results and joins.)
template <class S>
__device__ __forceinline__ Plan plan_of(const PageParams& p, const Counts& all, int most) {  // most: boxes of the longest head
  Plan plan = {0, 0, 0, all.boxes * p.subs};
  const int grid = gridDim.x;
  if (S::kWarpRows == kBoxRows && p.subs == 1 && p.own_queries && (long long)most * grid * kConsumers <= 2ll * all.boxes) {
    plan.by_warp = 1;
    plan.parts = grid;
  } else {
    // (a part is as long as a tile at least, so that a tile begins in it)
    plan.parts = min(grid, max(min(plan.total, 1), plan.total / kBoxesOf<S>));
    const bool whole = most <= 192 * 1024 / (2 * S::kBoxBytes);  // (bytes of a long head need not fit 32 bits)
    if (p.heads <= kPieceHeads)
#pragma unroll
      for (int i = kSizes - 1; i >= 0; --i) {
        const int n = all.of_size(i) * p.subs;
        const bool even = i < 3 || ((long long)kBoxesOf<S> * grid << (S::kPieceLog + i)) <= plan.total * 5ll / 2;
        if (i < 2 && plan.piece == 3 && whole) break;
        if (even && n <= min(i == 0 ? p.sms : grid, kMostPieces - 1)) {
          plan.piece = i + 1;
          plan.parts = n;
        }
      }
  }
  return plan;
}
// The line of `total` units in `parts` parts of equal size, the first total % parts of them one longer: where part i
// begins, and the part that unit u is in.
__device__ __forceinline__ int part_begin(int total, int parts, int i) {
  return total / parts * i + min(i, total % parts);
}
__device__ __forceinline__ int part_of(int total, int parts, int u) {
  const int size = total / parts, longer = total % parts;
  return u < longer * (size + 1) ? u / (size + 1) : longer + (u - longer * (size + 1)) / size;
}

// A CTA's part: its first tile, and where it ends.
struct Part {
  int head, sub, tile;   // head of the call, portion of its queries, tile in it
  int at, end;           // the line's box that the portion begins with, and the first one behind the part
  int first, pieces;     // of a piece: the portion's first piece and their number
};

// A portion that other CTAs have tiles of too: those from CTA w0 on, n of them (0: there is none).
struct Pending {
  int w0, n, queries;
  size_t q_row;
};

template <int D, bool BF16, int Q>
using WarpOf = typename std::conditional<BF16, TensorWarp<D, Q>, PlainWarp<D, Q>>::type;

constexpr int kFew = 8;     // CTAs whose results are joined straight from memory, at most
constexpr int kSegs = 64;  // segments of heads that are counted, at most

template <int D, bool BF16, int Q>
struct Shared {
  using S = Shape<D, BF16, Q>;
  using Warp = WarpOf<D, BF16, Q>;
  uint64_t full[S::kStages], empty[S::kStages], joined;
  uint64_t full_own[S::kStages][kConsumers];           // by warp: of its box of a stage
  Ctl ctl;
  int issued, last_one[2];
  Pending pending[2];                                  // the portions that the part begins and ends in
  Counts segs[kSegs];
  int2 seen[kThreads / 32];                            // by warp: boxes of the longest head, heads without rows
  float2 stats[kConsumers][Q];
  alignas(16) unsigned char q_mem[Warp::kOwnQueries ? kConsumers : 1][Warp::kQueryBytes];
  alignas(16) float probs[BF16 ? 1 : kConsumers][BF16 ? 4 : S::kWarpRows * Q];
};

// First row of the pool that the box of rows `row` ... of a head is in (a page that is none of the pool: behind the
// pool's rows, where copies give zeros).
__device__ __forceinline__ int place(const PageParams& p, int h, int row) {
  const Cache& c = p.c;
  const int page = p.table[(size_t)(p.first_head + h) * c.max_pages + (row >> c.page_shift)];
  return (unsigned)page < (unsigned)c.n_pages ? (page << c.page_shift) + (row & (c.page_rows - 1))
                                              : c.n_pages << c.page_shift;
}
// First row of the queries, and of the outputs, of a KV head: query heads lie in the order of their KV heads.
__device__ __forceinline__ size_t first_query(const Cache& c, int h) { return (size_t)h * c.group; }
// Inclusive prefix sum over the warp.
__device__ __forceinline__ int scan_warp(int x) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// The head that unit u of all heads' units is in, and how many units lie before that head; of_seg(i) and of_len(rows) say
// how many a segment and a head have.  For whole warps.
template <class OfSeg, class OfLen>
__device__ __forceinline__ int2 find_unit(const PageParams& p, int seg_heads, int u, OfSeg of_seg, OfLen of_len) {
  const int lane = threadIdx.x & 31;
  int at = 0, seg = 0;
  for (;; seg += 32) {
    const int mine = (seg + lane) * seg_heads < p.heads ? of_seg(seg + lane) : 0;
    const int upto = scan_warp(mine);
    const unsigned past = __ballot_sync(0xffffffffu, at + upto > u);
    if (past) {
      const int i = __ffs(past) - 1;
      at += __shfl_sync(0xffffffffu, upto - mine, i);
      seg += i;
      break;
    }
    at += __shfl_sync(0xffffffffu, upto, 31);
    if ((seg + 32) * seg_heads >= p.heads) return make_int2(p.heads, at);  // behind the last unit
  }
  for (int h = seg * seg_heads; h < p.heads; h += 32) {
    const int mine = h + lane < p.heads ? of_len(head_len(p, h + lane)) : 0;
    const int upto = scan_warp(mine);
    const unsigned past = __ballot_sync(0xffffffffu, at + upto > u);
    if (past) {
      const int i = __ffs(past) - 1;
      return make_int2(h + i, at + __shfl_sync(0xffffffffu, upto - mine, i));
    }
    at += __shfl_sync(0xffffffffu, upto, 31);
  }
  return make_int2(p.heads, at);
}

// One warp's heads [h, end) of `boxes` boxes in all, alone: it fetches its own boxes, a place in every stage.  32 boxes
// at a time are looked up, a lane each, and the next 32 while these are worked on.
template <int D, bool BF16, int Q>
__device__ __forceinline__ void whole_heads(const PageParams& p, const CUtensorMap* map_k, const CUtensorMap* map_v,
                                            Shared<D, BF16, Q>& sh, uint32_t ring, int h, int end, int boxes) {
  using S = Shape<D, BF16, Q>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned char* const q_mem = sh.q_mem[WarpOf<D, BF16, Q>::kOwnQueries ? warp : 0];
  WarpOf<D, BF16, Q> w;
  const Logit logit(p.c);
  struct Batch {
    int head, row, len, at;  // this lane's box
  };
  int next_head = h, next_row = 0;  // the first box that is not in a batch yet
  const auto look_up = [&] {
    Batch b = {end, 0, 0, 0};
    int n = 0;  // boxes in the batch
    while (n < 32 && next_head < end) {
      // boxes of the next 32 heads, counted on from those in hand
      const int len = next_head + lane < end ? head_len(p, next_head + lane) : 0;
      const int upto = scan_warp(boxes_of(len) - (lane == 0 ? next_row / kBoxRows : 0));
      const int want = lane - n;    // which of these boxes is this lane's
      int of = 0;                   // the head that it is in: as many heads end before it or with it
#pragma unroll
      for (int step = 16; step > 0; step >>= 1)
        if (__shfl_sync(0xffffffffu, upto, of + step - 1) <= want) of += step;
      const int all = __shfl_sync(0xffffffffu, upto, 31);
      const int ended = __shfl_sync(0xffffffffu, upto, max(0, of - 1)), before = of > 0 ? ended : 0;
      const int its_len = __shfl_sync(0xffffffffu, len, of);
      if (want >= 0 && want < all) {
        b.head = next_head + of;
        b.row = (want - before) * kBoxRows + (of == 0 ? next_row : 0);
        b.len = its_len;
      }
      const int took = min(32 - n, all);
      if (took < all) {  // the batch is full inside these heads
        const int lh = __shfl_sync(0xffffffffu, b.head, 31), lr = __shfl_sync(0xffffffffu, b.row, 31);
        const int ll = __shfl_sync(0xffffffffu, b.len, 31);
        next_head = lr + kBoxRows < ll ? lh : lh + 1;
        next_row = lr + kBoxRows < ll ? lr + kBoxRows : 0;
      } else {
        next_head = min(end, next_head + 32);
        next_row = 0;
      }
      n += took;
    }
    if (lane < n) b.at = place(p, b.head, b.row);
    return b;
  };
  Batch cur = look_up(), nxt = look_up();
  int sent = 0, first = 0;  // boxes asked for; number of the first of `cur`
  const auto send = [&] {
    const int i = sent - first;
    const int at = __shfl_sync(0xffffffffu, i < 32 ? cur.at : nxt.at, i & 31), stage = sent % S::kStages;
    const uint32_t bar = smem_u32(&sh.full_own[stage][warp]);
    if (lane == 0) mbar_expect_tx(bar, 2 * S::kBoxBytes);
    __syncwarp();
    if (lane < 2)
      tma_load_3d(ring + stage * S::kStageBytes + lane * S::kTileBytes + warp * S::kBoxBytes, lane ? map_v : map_k, 0, at, 0, bar);
    ++sent;
  };
  while (sent < min(boxes, S::kStages)) send();
  int in_hand = -1, fetched = -1;
  bool alive = true;
  for (int i = 0; i < boxes; ++i) {
    if (i - first == 32) {
      cur = nxt;
      first += 32;
      nxt = look_up();
    }
    const int head = __shfl_sync(0xffffffffu, cur.head, i - first), row = __shfl_sync(0xffffffffu, cur.row, i - first);
    const int len = __shfl_sync(0xffffffffu, cur.len, i - first), stage = i % S::kStages;
    if (head != in_hand) {
      if (fetched != head) w.fetch(p, first_query(p.c, head), p.c.group);
      w.begin(q_mem);
      in_hand = head;
      fetched = min(head + 1, p.heads - 1);  // the next head's, in case it follows
      w.fetch(p, first_query(p.c, fetched), p.c.group);
    }
    alive = __all_sync(0xffffffffu, wait_bar(smem_u32(&sh.full_own[stage][warp]), (i / S::kStages) & 1, &sh.ctl, p.status,
                                             true, p.sleep));
    if (!alive) break;
    const uint32_t k_tile = ring + stage * S::kStageBytes;
    w.tile(k_tile, k_tile + S::kTileBytes, warp * kBoxRows, min(kBoxRows, len - row), logit, q_mem,
           sh.probs[BF16 ? 0 : warp]);
    __syncwarp();
    if (sent < boxes) send();
    if (row + kBoxRows >= len) w.finish(p, first_query(p.c, head), p.c.group);
  }
  if (!alive && lane == 0)  // no warp leaves under a copy of its own
    for (int i = max(0, sent - S::kStages); i < sent; ++i)
      wait_bar(smem_u32(&sh.full_own[i % S::kStages][warp]), (i / S::kStages) & 1, &sh.ctl, p.status, false);
}

// The partial results of a portion's CTAs, joined in their order, by the consumer warps of the CTA that came last.
// The ring, which is at rest, takes them: all that fits is on its way at once, since a load takes 2 us while others use
// the memory.
template <int D, bool BF16, int Q>
__device__ __forceinline__ bool join_parts(const PageParams& p, Shared<D, BF16, Q>& sh, const Pending& x,
                                           unsigned char* ring_mem, int& turn) {
  using S = Shape<D, BF16, Q>;
  const int tid = threadIdx.x, n = x.n, queries = x.queries;
  const auto slot = [&](int i) { return (size_t)(x.w0 + i) * 2 + (i == 0); };  // (there the last, then the first portion)
  float2* const ml = reinterpret_cast<float2*>(ring_mem);                      // [query][part]
  const int head_bytes = (queries * n * 8 + 15) / 16 * 16, row_bytes = queries * D * 4;
  unsigned char* const rows = ring_mem + head_bytes;
  const int fit = (S::kStages * S::kStageBytes - head_bytes) / row_bytes;      // parts at a time
  // (the partial results and what the ring held before are there for the copies that follow)
  asm volatile("fence.proxy.async;" ::: "memory");
  meet();
  float4 acc[Q * D / 4 / (kConsumers * 32) + 1];
#pragma unroll
  for (int j = 0; j < (int)(sizeof(acc) / sizeof(acc[0])); ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0; i0 < n; i0 += fit) {
    const int cnt = min(fit, n - i0);
    if (i0 > 0) meet();
    if (tid < 32) {
      if (tid == 0) mbar_expect_tx(smem_u32(&sh.joined), cnt * row_bytes);
      __syncwarp();
      for (int i = tid; i < cnt; i += 32)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(smem_u32(rows + i * row_bytes)), "l"(p.part + slot(i0 + i) * Q * D), "r"(row_bytes),
                       "r"(smem_u32(&sh.joined)) : "memory");
    }
    if (i0 == 0) {
      for (int e = tid; e < n * queries; e += kConsumers * 32) {
        const int i = e / queries, q = e - i * queries;
        ml[q * n + i] = __ldcg(p.part_ml + slot(i) * Q + q);
      }
      meet();
      // maxima to weights; the weighted sum of the sums in front
      for (int q = tid >> 5; q < queries; q += kConsumers) {
        const int lane = tid & 31;
        float top = -INFINITY, l = 0.f;
        for (int i = lane; i < n; i += 32) top = fmaxf(top, ml[q * n + i].x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        for (int i = lane; i < n; i += 32) {
          const float e = fast_exp2(ml[q * n + i].x - finite_ref(top));
          l = fmaf(e, ml[q * n + i].y, l);
          ml[q * n + i].x = e;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        __syncwarp();
        if (lane == 0) {
          ml[q * n].y = l;
          if (p.lse) p.lse[x.q_row + q] = (top + fast_log2(l)) * kLn2;
        }
      }
    }
    if (!meet_all(wait_bar(smem_u32(&sh.joined), turn++ & 1, &sh.ctl, p.status, false))) return false;
#pragma unroll
    for (int j = 0; j < (int)(sizeof(acc) / sizeof(acc[0])); ++j) {
      const int e = tid + j * kConsumers * 32;
      if (e >= queries * (D / 4)) break;
      const int q = e / (D / 4);
#pragma unroll 4
      for (int i = 0; i < cnt; ++i) {
        const float w = ml[q * n + i0 + i].x;
        const float4 f = *reinterpret_cast<const float4*>(rows + (size_t)i * row_bytes + e * 16);
        acc[j] = make_float4(fmaf(w, f.x, acc[j].x), fmaf(w, f.y, acc[j].y), fmaf(w, f.z, acc[j].z), fmaf(w, f.w, acc[j].w));
      }
    }
  }
#pragma unroll
  for (int j = 0; j < (int)(sizeof(acc) / sizeof(acc[0])); ++j) {
    const int e = tid + j * kConsumers * 32;
    if (e >= queries * (D / 4)) break;
    const int q = e / (D / 4);
    const float l = ml[q * n].y;
    store4<BF16>(p.out, (x.q_row + q) * D + e % (D / 4) * 4, make_float4(acc[j].x / l, acc[j].y / l, acc[j].z / l, acc[j].w / l));
  }
  if (tid == 0) p.counters[x.w0] = 0;  // ready for the next call
  return true;
}

// The same for few CTAs, straight from memory: a thread has four columns of a query and loads them of all CTAs at once.
template <int D, bool BF16, int Q>
__device__ __forceinline__ void join_few(const PageParams& p, const Pending& x) {
  const int n = x.n;
  const auto slot = [&](int i) { return (size_t)(x.w0 + i) * 2 + (i == 0); };
  for (int e = threadIdx.x; e < x.queries * (D / 4); e += kConsumers * 32) {
    const int q = e / (D / 4), col = e % (D / 4) * 4;
    float2 ml[kFew];
    float4 f[kFew];
#pragma unroll
    for (int i = 0; i < kFew; ++i) {
      ml[i] = i < n ? __ldcg(p.part_ml + slot(i) * Q + q) : make_float2(-INFINITY, 0.f);
      f[i] = i < n ? __ldcg(reinterpret_cast<const float4*>(p.part + (slot(i) * Q + q) * D + col)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float top = ml[0].x;
#pragma unroll
    for (int i = 1; i < kFew; ++i) top = fmaxf(top, ml[i].x);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < kFew; ++i) {
      const float w = fast_exp2(ml[i].x - finite_ref(top));
      a = make_float4(fmaf(w, f[i].x, a.x), fmaf(w, f[i].y, a.y), fmaf(w, f[i].z, a.z), fmaf(w, f[i].w, a.w));
      l = fmaf(w, ml[i].y, l);
    }
    store4<BF16>(p.out, (x.q_row + q) * D + col, make_float4(a.x / l, a.y / l, a.z / l, a.w / l));
    if (p.lse && col == 0) p.lse[x.q_row + q] = (top + fast_log2(l)) * kLn2;
  }
  if (threadIdx.x == 0) p.counters[x.w0] = 0;  // ready for the next call
}

template <int D, bool BF16, int Q>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
decode_pages_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ PageParams p) {
  using S = Shape<D, BF16, Q>;
  using Warp = WarpOf<D, BF16, Q>;
  constexpr int kWarpsAll = kThreads / 32;
  extern __shared__ unsigned char smem_raw[];
  __shared__ Shared<D, BF16, Q> sh;
  const Cache& c = p.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* const ring_mem = smem_raw + (ring - smem_u32(smem_raw));

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v));
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(smem_u32(&sh.full[s]), 1);
      mbar_init(smem_u32(&sh.empty[s]), kConsumers);
      for (int w = 0; w < kConsumers; ++w) mbar_init(smem_u32(&sh.full_own[s][w]), 1);
    }
    mbar_init(smem_u32(&sh.joined), 1);
    sh.ctl.abort_flag = 0;
    sh.ctl.wait_cycles = p.wait_cycles;
    sh.issued = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  in_stream_order();

  // ---- the cut: segments of heads are counted, a warp each; every warp finds what it needs ----------
  int seg_heads = 32;  // a power of two
  while (seg_heads * kSegs < p.heads) seg_heads *= 2;
  // (Little code for few heads: it is fetched anew by every launch.)
  int most = 0, empty = 0;  // boxes of the longest head, heads without rows
  const auto see = [&](int len) {
    most = max(most, boxes_of(len));
    empty += len == 0;
    return len;
  };
  if (p.heads <= kPieceHeads) {
    for (int seg = warp; 32 * seg < p.heads; seg += kWarpsAll) {
      const int h = 32 * seg + lane;
      const Counts sum = Counts::of<S>(h < p.heads ? see(head_len(p, h)) : 0).over_warp();
      if (lane == 0) sh.segs[seg] = sum;
    }
  } else {
    const int span = max(512, seg_heads), per_seg = seg_heads / 32;
    for (int h0 = warp * span; h0 < p.heads; h0 += kWarpsAll * span) {
      int mine = 0;
      for (int i = h0; i < h0 + span; i += 512) {
        int len[16];  // sixteen loads at once
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int h = i + 32 * j + lane;
          len[j] = h < p.heads ? head_len(p, h) : -1;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (len[j] >= 0) mine += boxes_of(see(len[j]));
          const int h = i + 32 * j;
          if (((h / 32 + 1) & (per_seg - 1)) == 0) {
            const int sum = __reduce_add_sync(0xffffffffu, mine);
            if (lane == 0 && h - (seg_heads - 32) < p.heads) sh.segs[h / seg_heads].boxes = sum;
            mine = 0;
          }
        }
      }
    }
  }
  most = __reduce_max_sync(0xffffffffu, most);
  empty = __reduce_add_sync(0xffffffffu, empty);
  if (lane == 0) sh.seen[warp] = make_int2(most, empty);
  __syncthreads();
  Counts all = {};
  for (int seg = lane; seg * seg_heads < p.heads; seg += 32) {
    all.boxes += sh.segs[seg].boxes;
    if (p.heads <= kPieceHeads)  // (that is one segment a lane)
#pragma unroll
      for (int i = 0; i < kSizes / 2; ++i) all.pieces[i] = sh.segs[seg].pieces[i];
  }
  all = all.over_warp();
#pragma unroll
  for (int w = 0; w < kWarpsAll; ++w) {
    most = max(most, sh.seen[w].x);
    empty |= sh.seen[w].y;
  }
  if (empty)  // zeros for heads without rows
    for (int h = blockIdx.x + tid * gridDim.x; h < p.heads; h += kThreads * gridDim.x) {
      if (head_len(p, h) > 0) continue;
      const size_t row = first_query(c, h);
      for (int e = 0; e < c.group * D; e += 4) store4<BF16>(p.out, row * D + e, make_float4(0.f, 0.f, 0.f, 0.f));
      if (p.lse)
        for (int e = 0; e < c.group; ++e) p.lse[row + e] = -INFINITY;
    }
  const Plan plan = plan_of<S>(p, all, most);
  if ((int)blockIdx.x >= plan.parts) return;

  if (plan.by_warp) {
    if constexpr (S::kWarpRows == kBoxRows && Warp::kOwnQueries) {
      if (warp == kConsumers) return;
      // the heads whose first box is in this warp's part of all boxes
      const int workers = plan.parts * kConsumers, i = blockIdx.x * kConsumers + warp;
      int begin[2], at[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int cut = part_begin(all.boxes, workers, i + k);
        const int2 f = find_unit(p, seg_heads, cut, [&](int i) { return sh.segs[i].boxes; }, boxes_of);
        begin[k] = f.x;
        at[k] = f.y;
        if (f.y < cut && f.x < p.heads) {  // inside a head: the next one
          at[k] += boxes_of(head_len(p, f.x));
          ++begin[k];
        }
      }
      whole_heads(p, &map_k, &map_v, sh, ring, begin[0], begin[1], at[1] - at[0]);
    }
    return;
  }
  Part part;
  {
    // the piece, or the box, that this CTA's part begins with
    const int unit = plan.piece ? (int)blockIdx.x : part_begin(plan.total, plan.parts, blockIdx.x);
    const auto of_len = [&](int len) { return plan.piece ? Counts::pieces_of<S>(len, plan.piece - 1) : boxes_of(len); };
    const int2 f = find_unit(p, seg_heads, unit,
                             [&](int i) { return (plan.piece ? sh.segs[i].of_size(plan.piece - 1) : sh.segs[i].boxes) * p.subs; },
                             [&](int len) { return of_len(len) * p.subs; });
    if (f.x >= p.heads) return;  // (only where row counts have changed since they were counted, which no caller may do)
    const int len = head_len(p, f.x), tiles = tiles_of<S>(len), n = of_len(len);
    const int sub = p.subs == 1 ? 0 : (unit - f.y) / n, i = unit - f.y - sub * n;
    if (plan.piece) {
      // (a line of its own, which ends with the piece)
      const int t0 = n == 1 ? 0 : part_begin(tiles, n, i), t1 = n == 1 ? tiles : part_begin(tiles, n, i + 1);
      part = {f.x, sub, t0, 0, min(boxes_of(len), t1 * kBoxesOf<S>), unit - i, n};
    } else {
      // the first tile that begins there or behind it: it may be the next portion's
      part = {f.x, sub, (i + kBoxesOf<S> - 1) / kBoxesOf<S>, f.y + sub * n, part_begin(plan.total, plan.parts, blockIdx.x + 1), 0, 0};
    }
  }
  const auto wait = [&](uint64_t* bar, int parity) {  // the same in all lanes
    return __all_sync(0xffffffffu, wait_bar(smem_u32(bar), parity, &sh.ctl, p.status, true, p.sleep)) != 0;
  };
  int stage = 0, parity = 0;
  const auto next_stage = [&] {
    if (++stage == S::kStages) {
      stage = 0;
      parity ^= 1;
    }
  };
  // the portion in hand: its head, where it begins on the line, its first tile that is this CTA's
  int h = part.head, sub = part.sub, at0 = part.at, t0 = part.tile;

  if (warp == kConsumers) {
    // ---- producer ----------------------------------------------------------------------------------
    constexpr int kBoxes = kBoxesOf<S>, kAhead = 32 / kBoxes;
    int done = 0;  // tiles
    bool alive = true;
    for (; at0 < part.end && alive && h < p.heads; ++h, sub = 0) {
      const int len = head_len(p, h), n = tiles_of<S>(len), its_boxes = boxes_of(len);
      if (n == 0) continue;
      for (; sub < p.subs && at0 < part.end && alive; ++sub, t0 = 0, at0 += its_boxes) {
        const int tiles = min(n, (part.end - at0 + kBoxes - 1) / kBoxes) - t0;
        if (tiles <= 0) continue;
        int places = 0;
        for (int t = 0; t < tiles; ++t) {
          if (t % kAhead == 0) {  // the places of the next 32 boxes, a lane each
            const int row = (t0 + t) * S::kTile + lane * kBoxRows;
            places = row < len ? place(p, h, row) : 0;
          }
          const int boxes = min(kBoxes, (len - (t0 + t) * S::kTile + kBoxRows - 1) / kBoxRows);
          // lane 2 i + v: box i of K or V
          const int at = __shfl_sync(0xffffffffu, places, t % kAhead * kBoxes + (lane >> 1) % kBoxes);
          if (done + t >= S::kStages && !(alive = wait(&sh.empty[stage], parity ^ 1))) break;
          if (lane == 0) {
            mbar_expect_tx(smem_u32(&sh.full[stage]), 2 * boxes * S::kBoxBytes);
            ++sh.issued;
          }
          __syncwarp();
          if (lane < 2 * boxes) {
            const bool v = lane & 1;
            tma_load_3d(ring + stage * S::kStageBytes + (v ? S::kTileBytes : 0) + (lane >> 1) * S::kBoxBytes,
                        v ? &map_v : &map_k, 0, at, 0, smem_u32(&sh.full[stage]));
          }
          next_stage();
        }
        done += tiles;
      }
    }
  } else {
    // ---- consumers ---------------------------------------------------------------------------------
    Warp w;
    const Logit logit(c);
    unsigned char* const q_mem = sh.q_mem[Warp::kOwnQueries ? warp : 0];
    float* const probs = sh.probs[BF16 ? 0 : warp];
    int fetched = -1;  // the head whose queries are on their way
    bool alive = true, begun = false, ended = false;  // others have tiles of the portion that the part begins, ends in
    for (; at0 < part.end && alive && h < p.heads; ++h, sub = 0) {
      const int len = head_len(p, h), n = tiles_of<S>(len), its_boxes = boxes_of(len);
      if (n == 0) continue;
      for (; sub < p.subs && at0 < part.end; ++sub, t0 = 0, at0 += its_boxes) {
        const int tiles = min(n, (part.end - at0 + kBoxesOf<S> - 1) / kBoxesOf<S>) - t0;
        if (tiles <= 0) continue;
        const int queries = min(p.per_sub, c.group - sub * p.per_sub);
        if (fetched != h) w.fetch(p, first_query(c, h) + sub * p.per_sub, queries);
        w.begin(q_mem);
        if (p.subs == 1) {  // the next head's, in case it follows
          fetched = min(h + 1, p.heads - 1);
          w.fetch(p, first_query(c, fetched), queries);
        }
        int valid = len - t0 * S::kTile - warp * S::kWarpRows;  // rows from this warp's first one on
        for (int t = 0;; ++t, valid -= S::kTile) {
          const uint32_t k_tile = ring + stage * S::kStageBytes;
          if (!(alive = wait(&sh.full[stage], parity))) break;
          if (valid > 0)
            w.tile(k_tile, k_tile + S::kTileBytes, warp * S::kWarpRows, min(S::kWarpRows, valid), logit, q_mem, probs);
          if (t + 1 == tiles) break;  // (the last stage is kept for the meeting)
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sh.empty[stage]));
          next_stage();
        }
        // The warps meet: each leaves its maxima and sums, and what it has summed of V in the memory of its own rows of
        // the last stage, which no other warp reads.
        unsigned char* const last = ring_mem + stage * S::kStageBytes;
        w.leave_stats(sh.stats[warp]);
        __syncwarp();
        w.leave_sums(last, warp);
        alive = meet_all(alive);
        if (!alive) break;
        const size_t q_row = first_query(c, h) + sub * p.per_sub;
        const bool whole = tiles == n;
        const size_t slot = (size_t)blockIdx.x * 2 + (t0 == 0);
        for (int e = tid; e < queries * (D / 4); e += kConsumers * 32) {
          const int q = e / (D / 4), col = e % (D / 4) * 4;
          const float top = top_of<Q>(sh.stats, q);
          float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
          float l = 0.f;
#pragma unroll
          for (int i = 0; i < kConsumers; ++i) {
            const float4 f = *reinterpret_cast<const float4*>(last + Warp::sum_at(i, q, col));
            const float x = fast_exp2(sh.stats[i][q].x - finite_ref(top));
            a = make_float4(fmaf(f.x, x, a.x), fmaf(f.y, x, a.y), fmaf(f.z, x, a.z), fmaf(f.w, x, a.w));
            l = fmaf(sh.stats[i][q].y, x, l);
          }
          if (whole) {
            store4<BF16>(p.out, (q_row + q) * D + col, make_float4(a.x / l, a.y / l, a.z / l, a.w / l));
            if (p.lse && col == 0) p.lse[q_row + q] = (top + fast_log2(l)) * kLn2;
          } else {
            *reinterpret_cast<float4*>(p.part + (slot * Q + q) * D + col) = a;
            if (col == 0) p.part_ml[slot * Q + q] = make_float2(top, l);
          }
        }
        if (!whole) {
          if (t0 == 0) ended = true;
          else begun = true;
          if (tid == 0) {  // the CTAs that have tiles of the portion
            Pending x = {part.first, part.pieces, queries, q_row};
            if (!plan.piece) {
              x.w0 = part_of(plan.total, plan.parts, at0);
              x.n = part_of(plan.total, plan.parts, at0 + (n - 1) * kBoxesOf<S>) + 1 - x.w0;
            }
            sh.pending[t0 == 0] = x;
          }
        }
        fence_async_proxy();  // (the stage was written; the next copy into it comes after)
        meet();
        if (lane == 0) mbar_arrive(smem_u32(&sh.empty[stage]));
        next_stage();
      }
    }
    // Portions that other CTAs have tiles of, when the part is through: who comes last joins them.
    if (alive && (begun || ended)) {
      asm volatile("fence.proxy.async;" ::: "memory");  // (bulk copies will read the partial results)
      __threadfence();
      meet();
      if (tid == 0 && begun) sh.last_one[0] = atomicAdd(p.counters + sh.pending[0].w0, 1) == sh.pending[0].n - 1;
      if (tid == 32 && ended) sh.last_one[1] = atomicAdd(p.counters + sh.pending[1].w0, 1) == sh.pending[1].n - 1;
      meet();
      __threadfence();
      int turn = 0;
      for (int i = begun ? 0 : 1; i < (ended ? 2 : 1); ++i)
        if (sh.last_one[i]) {
          const Pending x = sh.pending[i];
          if (x.n <= kFew) join_few<D, BF16, Q>(p, x);
          else if (!join_parts(p, sh, x, ring_mem, turn)) break;
        }
    }
  }
  // after a wait that gave up: no CTA leaves under a copy of its own
  __syncthreads();
  if (sh.ctl.abort_flag && tid == 0) {
    for (int i = max(0, sh.issued - S::kStages); i < sh.issued; ++i) {
      wait_bar(smem_u32(&sh.full[i % S::kStages]), (i / S::kStages) & 1, &sh.ctl, p.status, false);
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
  static std::atomic<unsigned long long> told{0};  // devices that know how much shared memory the kernel takes
  int dev = 0;
  lava_status rc = check_cuda(cudaGetDevice(&dev), "current device");
  if (rc != LAVA_OK) return rc;
  if (dev >= 64 || !(told.load(std::memory_order_relaxed) >> dev & 1)) {
    rc = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem),
                    "paged decode attention attribute");
    if (rc != LAVA_OK) return rc;
    if (dev < 64) told.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  const long long most = ((((long long)p.c.max_pages << p.c.page_shift) + S::kTile - 1) / S::kTile) * p.heads * p.subs;
  const int grid = (int)std::min<long long>(most_ctas(), most);
  p.own_queries = WarpOf<D, BF16, Q>::kOwnQueries;
  p.sms = most_ctas() / kCtasPerSm;
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
  const size_t need = lava_cache_workspace_bytes(cache);
  if (!workspace || workspace_bytes < need)
    return fail(LAVA_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
  if (!aligned16(workspace)) return fail(LAVA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  const Portions portions = portions_of(c);
  if ((long long)n_layers * c.batch * c.n_kv_heads * portions.subs >= (1ll << 35) / ((long long)c.max_pages << c.page_shift))
    return fail(LAVA_ERR_UNSUPPORTED, "too many rows in one call: heads * max_pages * page_rows must stay below 2^35");
  // blocks read queries while others write outputs
  const size_t io_bytes = (size_t)n_layers * c.batch * c.n_q_heads * c.head_dim * (c.dtype == LAVA_BF16 ? 2 : 4);
  if ((const char*)q < (const char*)out + io_bytes && (const char*)out < (const char*)q + io_bytes)
    return fail(LAVA_ERR_INVALID_ARG, "out overlaps q");
  CUtensorMap map_k, map_v;
  rc = encode_pages_map(c, k_pages, &map_k);
  if (rc == LAVA_OK) rc = encode_pages_map(c, v_pages, &map_v);
  if (rc != LAVA_OK) return rc;
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
  p.sleep = p.wait_cycles >= 4000;
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
