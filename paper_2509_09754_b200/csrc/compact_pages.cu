// Gather of the retained K/V rows into the pages of a paged cache.
//
// The rows of all (layer, sequence, KV head) in their order are one line, which is cut into equal runs of consecutive
// rows, a run per warp: heads keep uneven numbers of rows (up to eight times the mean), and with blocks per head, as
// the packed compaction has them, the longest is waited for.  Blocks per head / runs, us on the device, one prompt again
// and again: 32 layers x 32K, 524288 rows 110 / 95; 8K, 131072 rows 35.5 / 21.7; 1K, 32768 rows 9.6 / 7.4; ragged batch of
// 8, 262144 rows 52.8 / 52.7.  (Runs, several prompts in turn, so that nothing of one is in L2: 96, 28.5, 8.1.)  Row
// counts live on the device, so every warp finds its run itself, from the rows of the problems (layer, sequence).
//
// A lane looks up a row: its head, its position (kept list or window), its page; for the next 32 rows while these are
// moved.  Then 8, 16 or 32 lanes copy a row with 16-byte accesses, several rows at once.
//
// Bound by HBM: every row is read and written once, in scattered rows of 128 to 512 bytes (5.6 TB/s where a copy has
// 6.6).  Three blocks per SM with two passes at once: more of either and the scattered reads get in one another's way
// (32K: four blocks of four passes 101 us, six of two 105; runs dealt out in turns of 32 rows 102); reads that are not
// kept in the cache 95 against 98.
#include <algorithm>

#include "lava_internal.cuh"

namespace lava {
namespace {

constexpr int kThreads = 256;
constexpr int kBlocksPerSm = 3;

struct FillParams {
  Geom g;
  Cache c;
  int first_seq, problems;
  const char* k;
  const char* v;
  long long k_ls, v_ls;     // strides of layers, in elements
  const int* keep_idx;
  const int* head_offsets;  // [layers, batch, H_kv + 1]
  const int* first_row;     // [layers, batch, H_kv]
  const int* page_table;
  char* k_pages;
  char* v_pages;
};

// What a lane knows of its row: KV head, token (in the concatenated axis) and place in the pool (-1: it is not moved).
struct Row {
  int kvh, tok, place;
};

__device__ __forceinline__ Row look_up(const FillParams& p, int prob, const SeqInfo& s, int r, int rows) {
  const Geom& g = p.g;
  Row x = {0, 0, -1};
  if (r >= rows) return x;
  const int* hoff = p.head_offsets + (size_t)prob * (g.n_kv_heads + 1);
  int lo = 0, hi = g.n_kv_heads - 1;  // the head: the first one that ends behind row r
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (hoff[mid + 1] > r) hi = mid; else lo = mid + 1;
  }
  const int h0 = hoff[lo], win = min(g.window, s.n), j = r - h0, kept = hoff[lo + 1] - h0 - win;
  const int layer = prob / g.batch;
  x.kvh = lo;
  x.tok = (int)s.tok0 + (j < kept ? p.keep_idx[(size_t)layer * g.total_scores + s.score_off + (r - lo * win)]
                                  : s.prefix + (j - kept));
  const int first = p.first_row[(size_t)prob * g.n_kv_heads + lo];
  if (first >= 0 && j < (p.c.max_pages << p.c.page_shift) - first) {
    const int row = first + j, seq = p.first_seq + prob - layer * g.batch;
    const size_t head = ((size_t)layer * p.c.batch + seq) * p.c.n_kv_heads + lo;
    const int page = p.page_table[head * p.c.max_pages + (row >> p.c.page_shift)];
    if ((unsigned)page < (unsigned)p.c.n_pages) x.place = (page << p.c.page_shift) + (row & (p.c.page_rows - 1));
  }
  return x;
}

template <int RowBytes>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
compact_pages_kernel(const __grid_constant__ FillParams p) {
  in_stream_order();
  const Geom& g = p.g;
  if (batch_has_short_sequence(g)) return;  // the score layout has no room for such a batch
  constexpr int kLanes = RowBytes / 16, kRows = 32 / kLanes, kAhead = 2;  // lanes per row, rows per pass, passes at once
  const int lane = threadIdx.x & 31, sub = lane / kLanes, c = lane % kLanes;
  const int worker = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), workers = gridDim.x * (kThreads / 32);

  // ---- this warp's run ------------------------------------------------------------------------------
  const auto rows_of = [&](int prob) {
    return prob < p.problems ? max(0, p.head_offsets[(size_t)prob * (g.n_kv_heads + 1) + g.n_kv_heads]) : 0;
  };
  long long total = 0;
  for (int i = lane; i < p.problems; i += 32) total += rows_of(i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  const long long run = max((long long)kAhead * kRows, (total + workers - 1) / workers);
  long long at = worker * run;
  const long long end = min(total, at + run);
  if (at >= end) return;
  int prob = 0;
  long long before = 0;  // rows of the problems before it
  for (;; prob += 32) {
    const int mine = rows_of(prob + lane);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, before + upto > at);
    if (past) {
      const int i = __ffs(past) - 1;
      before += __shfl_sync(0xffffffffu, upto - mine, i);
      prob += i;
      break;
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }

  // ---- its rows, problem by problem -----------------------------------------------------------------
  for (; at < end; ++prob) {
    const int rows = rows_of(prob);
    const int layer = prob / g.batch;
    const SeqInfo s = seq_info(g, prob - layer * g.batch);
    const int first = (int)(at - before), last = (int)min((long long)rows, end - before);
    const int bytes = g.dtype == LAVA_BF16 ? 2 : 4;
    const char* kl = p.k + (long long)layer * p.k_ls * bytes + c * 16;
    const char* vl = p.v + (long long)layer * p.v_ls * bytes + c * 16;
    Row next = look_up(p, prob, s, first + lane, last);
    for (int r0 = first; r0 < last; r0 += 32) {
      const Row row = next;
      next = look_up(p, prob, s, r0 + 32 + lane, last);
#pragma unroll 1
      for (int i0 = 0; i0 < 32; i0 += kAhead * kRows) {
        if (r0 + i0 >= last) break;
        uint4 kk[kAhead], vv[kAhead];
        int place[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int i = i0 + u * kRows + sub;
          place[u] = __shfl_sync(0xffffffffu, row.place, i);
          const int kvh = __shfl_sync(0xffffffffu, row.kvh, i), tok = __shfl_sync(0xffffffffu, row.tok, i);
          if (place[u] >= 0) {
            kk[u] = __ldcs(reinterpret_cast<const uint4*>(kl + (kvh * g.k_sh + tok * g.k_st) * bytes));
            vv[u] = __ldcs(reinterpret_cast<const uint4*>(vl + (kvh * g.v_sh + tok * g.v_st) * bytes));
          }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (place[u] >= 0) {
            *reinterpret_cast<uint4*>(p.k_pages + (long long)place[u] * RowBytes + c * 16) = kk[u];
            *reinterpret_cast<uint4*>(p.v_pages + (long long)place[u] * RowBytes + c * 16) = vv[u];
          }
      }
    }
    at = before + last;
    before += rows;
  }
}

}  // namespace

lava_status launch_compact_pages(const Geom& g, const Cache& c, int first_seq, const void* k, const void* v,
                                 long long k_ls, long long v_ls, const int* keep_idx, const int* head_offsets,
                                 const int* first_row, const int* page_table, void* k_pages, void* v_pages,
                                 cudaStream_t stream) {
  FillParams p;
  p.g = g;
  p.c = c;
  p.first_seq = first_seq;
  p.problems = c.n_layers * g.batch;
  p.k = (const char*)k;
  p.v = (const char*)v;
  p.k_ls = k_ls;
  p.v_ls = v_ls;
  p.keep_idx = keep_idx;
  p.head_offsets = head_offsets;
  p.first_row = first_row;
  p.page_table = page_table;
  p.k_pages = (char*)k_pages;
  p.v_pages = (char*)v_pages;
  const int row_bytes = g.head_dim * (g.dtype == LAVA_BF16 ? 2 : 4);
  const auto kernel = row_bytes == 128 ? compact_pages_kernel<128>
                                       : row_bytes == 256 ? compact_pages_kernel<256> : compact_pages_kernel<512>;
  const int sms = sm_count() > 0 ? sm_count() : 148;
  const cudaError_t e = launch_in_order(kernel, sms * kBlocksPerSm, kThreads, 0, stream, p);
  count_launches(1);
  return check_cuda(e, "compact_kv_pages launch");
}

}  // namespace lava
