// Paged cache: descriptors, and the page tables of heads that get rows or give their pages back.
//
// A head (layer, sequence, KV head) with r rows holds ceil(r / page_rows) pages.  The heads that grow take
// the next free pages of the ring in the order of the heads; where a head's pages start is therefore an
// exclusive prefix sum of what the heads before it need, and so is the place of the pages that go back.
// Whether all can be served has to be known before anything is written.
//
// One cluster: a CTA takes a range of consecutive heads, sums what they need and give, the CTAs read one
// another's sums behind one cluster barrier, and each writes what its heads get.  Bound by latency: counters
// and counts, barrier, ring, table.  A token of 8 sequences in 32 layers of 8 heads: 5.8 us; four prompts of 2048 rows a
// head there, 32768 pages, 9.2; 5 and 32 rows a sequence, whose slots a head's thread writes in turn, 6.9 and 9.5.
#include <algorithm>

#include <cooperative_groups.h>

#include "lava_internal.cuh"

namespace lava {

lava_status make_cache(const lava_cache_desc* d, Cache* out) {
  if (!d) return fail(LAVA_ERR_INVALID_ARG, "cache is NULL");
  if (d->n_layers < 1 || d->batch < 1) return fail(LAVA_ERR_INVALID_ARG, "n_layers and batch must be >= 1");
  if (d->n_kv_heads < 1 || d->n_q_heads < 1 || d->n_q_heads % d->n_kv_heads != 0)
    return fail(LAVA_ERR_INVALID_ARG, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)",
                d->n_q_heads, d->n_kv_heads);
  if (d->n_kv_heads > 128) return fail(LAVA_ERR_UNSUPPORTED, "n_kv_heads > 128");
  if (d->n_q_heads > 65535) return fail(LAVA_ERR_UNSUPPORTED, "n_q_heads > 65535");
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(LAVA_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", d->head_dim);
  if (d->dtype != LAVA_F32 && d->dtype != LAVA_BF16)
    return fail(LAVA_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if (d->page_rows != 16 && d->page_rows != 32 && d->page_rows != 64 && d->page_rows != 128 &&
      d->page_rows != 256)
    return fail(LAVA_ERR_UNSUPPORTED, "page_rows must be 16, 32, 64, 128 or 256 (got %d)", d->page_rows);
  if (d->max_pages < 1 || d->n_pages < 1)
    return fail(LAVA_ERR_INVALID_ARG, "max_pages and n_pages must be >= 1");
  if (d->n_pages > 0x7fffffffLL / d->page_rows || d->max_pages > 0x3fffffff / d->page_rows)
    return fail(LAVA_ERR_UNSUPPORTED, "rows of the pool must stay below 2^31, those of a head below 2^30");
  const long long heads = (long long)d->n_layers * d->batch * d->n_kv_heads;
  if ((long long)d->n_layers * d->batch > (1 << 24) || heads > (1 << 24))
    return fail(LAVA_ERR_UNSUPPORTED, "more than 2^24 heads");
  if (!(d->sm_scale >= 0.f) || !(d->softcap >= 0.f) || isinf(d->sm_scale) || isinf(d->softcap))
    return fail(LAVA_ERR_INVALID_ARG, "sm_scale and softcap must be finite and >= 0");
  Cache c;
  c.n_layers = d->n_layers;
  c.batch = d->batch;
  c.n_q_heads = d->n_q_heads;
  c.n_kv_heads = d->n_kv_heads;
  c.group = d->n_q_heads / d->n_kv_heads;
  c.head_dim = d->head_dim;
  c.dtype = d->dtype;
  c.page_rows = d->page_rows;
  c.page_shift = 0;
  while ((1 << c.page_shift) < d->page_rows) ++c.page_shift;
  c.max_pages = d->max_pages;
  c.n_pages = (int)d->n_pages;
  c.heads = (int)heads;
  c.scale = d->sm_scale > 0.f ? d->sm_scale : (float)(1.0 / sqrt((double)d->head_dim));
  c.softcap = d->softcap;
  // the factors that logits are multiplied by in the base-2 domain
  constexpr float kLog2e = 1.44269504f;
  if (isinf(c.scale * kLog2e) || isinf(c.softcap * kLog2e) || (c.softcap > 0.f && !isnormal(c.scale / c.softcap)))
    return fail(LAVA_ERR_INVALID_ARG, "sm_scale, softcap or their quotient leaves fp32");
  *out = c;
  return LAVA_OK;
}

namespace {

namespace cg = cooperative_groups;

constexpr int kMostThreads = 1024;
constexpr int kMostCtas = 8;

struct TableParams {
  Cache c;
  const int* head_offsets;  // admit: [n_layers, n_seqs, H_kv + 1]
  int first_seq, n_seqs;
  const int* add;           // extend: [batch]
  int max_add;
  const int* rows;
  int* rows_out;
  int* table;
  const int* ring;
  int* ring_out;
  const long long* counters;
  long long* counters_out;
  int* first_row;
  int* slots;
  unsigned* status;
};

// What a call does to a head: the pages that it holds, takes and gives back, its rows before and after.
struct Change {
  int held, take, give, before, after, bad;
};

__device__ __forceinline__ Change change_of(const TableParams& p, int h) {
  const Cache& c = p.c;
  Change x;
  x.before = p.rows[h];
  const int prob = h / c.n_kv_heads, g = h - prob * c.n_kv_heads, layer = prob / c.batch, b = prob - layer * c.batch;
  long long add = 0;
  bool ok = true;
  if (p.add) {
    add = p.add[b];
    ok = add <= p.max_add;
  } else if (b >= p.first_seq && b < p.first_seq + p.n_seqs) {
    const int* o = p.head_offsets + ((size_t)layer * p.n_seqs + (b - p.first_seq)) * (c.n_kv_heads + 1) + g;
    add = (long long)o[1] - o[0];
    ok = add >= 0;
  }
  const long long most = (long long)c.max_pages << c.page_shift;
  const bool release = p.add && add < 0;
  const long long after = release ? 0 : x.before + add;
  x.bad = !ok || x.before < 0 || x.before > most || after > most;
  x.after = (int)after;
  x.held = x.bad ? 0 : (x.before + c.page_rows - 1) >> c.page_shift;
  x.take = x.bad || release ? 0 : ((x.after + c.page_rows - 1) >> c.page_shift) - x.held;
  x.give = x.bad || !release ? 0 : x.held;
  return x;
}

struct Sums {
  long long take, give;
  int bad;
};

// Inclusive prefix sums over the block; the totals in *sum.  (Sums that do not fit 32 bits belong to refused calls.)
__device__ __forceinline__ int2 scan_block(int2 x, int2* warps, int2* sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const auto scan = [&](int2 a) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, a.x, o), z = __shfl_up_sync(0xffffffffu, a.y, o);
      if (lane >= o) a = make_int2(a.x + y, a.y + z);
    }
    return a;
  };
  x = scan(x);
  if (lane == 31) warps[warp] = x;
  __syncthreads();
  const int2 upto = scan(lane < n_warps ? warps[lane] : make_int2(0, 0));
  *sum = make_int2(__shfl_sync(0xffffffffu, upto.x, 31), __shfl_sync(0xffffffffu, upto.y, 31));
  const int y = __shfl_sync(0xffffffffu, upto.x, max(0, warp - 1)), z = __shfl_sync(0xffffffffu, upto.y, max(0, warp - 1));
  __syncthreads();  // (the warps' sums are written again)
  return warp ? make_int2(x.x + y, x.y + z) : x;
}

// Entry i of the ring, counted from `start` (both below the ring's length).
__device__ __forceinline__ int ring_at(int start, int i, int n) {
  const int at = start + i;
  return at < n ? at : at - n;
}

// The pages that a head takes from the ring (n > 0) or gives back (n < 0), and where they lie in ring and table.
struct Move {
  int n, ring, table;
};
// Moves page numbers `first`, `first + step` ... of a head, U at a time: all loads before the stores, which might be to the
// same memory for all the compiler knows.
template <int U>
__device__ __forceinline__ void move_pages(const TableParams& p, int h, const Move& m, int first, int step) {
  int* const row = p.table + (size_t)h * p.c.max_pages + m.table;
  const int n = abs(m.n);
  for (int i0 = first; i0 < n; i0 += U * step) {
    int x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * step;
      x[u] = i >= n ? 0 : m.n > 0 ? p.ring[ring_at(m.ring, i, p.c.n_pages)] : row[i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * step;
      if (i >= n) break;
      if (m.n > 0) row[i] = x[u];
      else p.ring_out[ring_at(m.ring, i, p.c.n_pages)] = x[u];
    }
  }
}

__global__ void __launch_bounds__(kMostThreads)
page_table_kernel(const __grid_constant__ TableParams p) {
  in_stream_order();
  __shared__ int2 warps[32];
  __shared__ long long take_sums[32], give_sums[32];
  __shared__ Sums mine;
  // heads that move more than two pages: eight lanes move one, since a warp's heads may be of one prompt, and the others'
  // of none
  __shared__ int n_many, many[kMostThreads];
  __shared__ Move moves[kMostThreads];
  const Cache& c = p.c;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, ctas = gridDim.x, rank = blockIdx.x;
  const int share = (c.heads + ctas - 1) / ctas;
  const int h0 = min(c.heads, rank * share), h1 = min(c.heads, h0 + share);
  if (tid == 0) n_many = 0;
  const long long taken = p.counters[0], given = p.counters[1];

  // ---- what this CTA's heads need ---------------------------------------------------------------
  long long take = 0, give = 0;
  int bad = 0;
  Change first = {};  // of this thread's first head
  for (int h = h0 + tid; h < h1; h += threads) {
    const Change x = change_of(p, h);
    if (h < h0 + threads) first = x;
    take += x.take;
    give += x.give;
    bad |= x.bad;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    take += __shfl_xor_sync(0xffffffffu, take, o);
    give += __shfl_xor_sync(0xffffffffu, give, o);
  }
  if (lane == 0) {
    take_sums[warp] = take;
    give_sums[warp] = give;
  }
  bad = __syncthreads_or(bad);
  if (warp == 0) {
    take = lane < threads / 32 ? take_sums[lane] : 0;
    give = lane < threads / 32 ? give_sums[lane] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      take += __shfl_xor_sync(0xffffffffu, take, o);
      give += __shfl_xor_sync(0xffffffffu, give, o);
    }
    if (lane == 0) mine = {take, give, bad};
  }
  cluster.sync();
  long long take_at = 0, give_at = 0, take_all = 0, give_all = 0;
  bad = 0;
  for (int r = 0; r < ctas; ++r) {
    const Sums s = *cluster.map_shared_rank(&mine, r);
    if (r == rank) {
      take_at = take_all;
      give_at = give_all;
    }
    take_all += s.take;
    give_all += s.give;
    bad |= s.bad;
  }
  const bool short_of = taken < 0 || given < taken || given - taken > c.n_pages || take_all > given - taken;
  // (more pages given back than the pool has in use: the table and the counters do not belong together)
  if (!short_of && give_all > c.n_pages - (given - taken)) bad = 1;
  const bool refused = bad || short_of;
  // where this CTA's pages start in the ring
  int ring_take = refused ? 0 : (int)((taken + take_at) % c.n_pages), ring_give = refused ? 0 : (int)((given + give_at) % c.n_pages);

  // ---- what they get, a head per thread at a time -------------------------------------------------
  for (int at = h0; at < h1; at += threads) {
    const int h = at + tid;
    const bool live = h < h1;
    Change x = first;
    if (at > h0) x = live ? change_of(p, h) : Change{};
    if (!live) x = Change{};
    if (refused) x.take = x.give = 0;
    const int pages = x.take > 0 ? x.take : -x.give;
    const unsigned more = __ballot_sync(0xffffffffu, abs(pages) > 2);
    if (more) {
      int slot = 0;
      if (lane == 0) slot = atomicAdd(&n_many, __popc(more));
      slot = __shfl_sync(0xffffffffu, slot, 0) + __popc(more & ((1u << lane) - 1));
      if (more >> lane & 1) many[slot] = tid;
    }
    int2 sum;
    const int2 incl = scan_block(make_int2(x.take, x.give), warps, &sum);
    const int my_take = ring_at(ring_take, incl.x - x.take, c.n_pages);
    const size_t row = (size_t)h * c.max_pages;
    if (live) {
      p.rows_out[h] = refused ? x.before : x.after;
      const int prob = h / c.n_kv_heads, g = h - prob * c.n_kv_heads, layer = prob / c.batch, b = prob - layer * c.batch;
      if (p.first_row && b >= p.first_seq && b < p.first_seq + p.n_seqs)
        p.first_row[((size_t)layer * p.n_seqs + (b - p.first_seq)) * c.n_kv_heads + g] = refused ? -1 : x.before;
      if (p.slots) {
        const int n = refused ? 0 : max(0, x.after - x.before);
        for (int j = 0; j < p.max_add; ++j) {
          int slot = -1;
          if (j < n) {
            const int r = x.before + j, pg = r >> c.page_shift;
            const int page = pg < x.held ? p.table[row + pg] : p.ring[ring_at(my_take, pg - x.held, c.n_pages)];
            slot = page < 0 || page >= c.n_pages ? -1 : (page << c.page_shift) + (r & (c.page_rows - 1));
          }
          p.slots[((size_t)prob * p.max_add + j) * c.n_kv_heads + g] = slot;
        }
      }
    }
    const Move mine_here = {pages, pages > 0 ? my_take : ring_at(ring_give, incl.y - x.give, c.n_pages), pages > 0 ? x.held : 0};
    if (abs(pages) <= 2) move_pages<2>(p, h, mine_here, 0, 1);
    if (n_many > 0) {
      moves[tid] = mine_here;
      __syncthreads();
      for (int j = tid / 8; j < n_many; j += threads / 8) move_pages<4>(p, at + many[j], moves[many[j]], tid % 8, 8);
    }
    if (at + threads < h1) {  // (the list is made anew)
      __syncthreads();
      if (tid == 0) n_many = 0;
      __syncthreads();
    }
    ring_take = ring_at(ring_take, sum.x, c.n_pages);
    ring_give = ring_at(ring_give, sum.y, c.n_pages);
  }
  cluster.sync();  // every CTA has read the counters and the others' sums
  if (rank == 0 && tid == 0) {
    p.counters_out[0] = refused ? taken : taken + take_all;
    p.counters_out[1] = refused ? given : given + give_all;
    if (refused && p.status)
      atomicOr(p.status, (bad ? LAVA_DEV_BAD_ROWS : 0u) | (short_of ? LAVA_DEV_PAGES_EXHAUSTED : 0u));
  }
}

lava_status launch_tables(const TableParams& p, cudaStream_t stream) {
  if (reinterpret_cast<uintptr_t>(p.status) % 4 != 0)  // (it may be a word in a buffer of bytes)
    return fail(LAVA_ERR_INVALID_ARG, "status_word must be 4-byte aligned");
  // a CTA for every 128 heads and a thread per head, then more threads, then more heads per thread; for prompts, whose heads
  // take many pages, 512 threads at least (32768 pages of 1024 heads: 9.2 us, 256 threads 10.8, 1024 9.4; 4096 of 1024 heads
  // 6.5, 6.1, 7.8)
  int ctas = 1;
  while (ctas < kMostCtas && ctas * 128 < p.c.heads) ctas *= 2;
  const int share = (p.c.heads + ctas - 1) / ctas;
  const int threads = std::min(kMostThreads, std::max(p.add ? 0 : 512, (share + 31) / 32 * 32));
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = ctas;
  cfg.blockDim = threads;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, page_table_kernel, p);
  count_launches(1);
  return check_cuda(e, "page table launch");
}

}  // namespace
}  // namespace lava

using namespace lava;

extern "C" {

lava_status lava_page_admit(const lava_cache_desc* cache, int32_t first_seq, int32_t n_seqs,
                            const int32_t* head_offsets, const int32_t* head_rows, int32_t* head_rows_out,
                            int32_t* page_table, const int32_t* free_pages, const int64_t* counters,
                            int64_t* counters_out, int32_t* first_row, uint32_t* status_word, void* stream) {
  TableParams p = {};
  const lava_status rc = make_cache(cache, &p.c);
  if (rc != LAVA_OK) return rc;
  if (!head_offsets || !head_rows || !head_rows_out || !page_table || !free_pages || !counters || !counters_out ||
      !first_row)
    return fail(LAVA_ERR_INVALID_ARG, "NULL argument");
  if (n_seqs < 1 || first_seq < 0 || first_seq > p.c.batch - n_seqs)
    return fail(LAVA_ERR_INVALID_ARG, "sequences %d ... %lld are not all in a cache of %d", first_seq,
                (long long)first_seq + n_seqs - 1, p.c.batch);
  p.head_offsets = head_offsets;
  p.first_seq = first_seq;
  p.n_seqs = n_seqs;
  p.rows = head_rows;
  p.rows_out = head_rows_out;
  p.table = page_table;
  p.ring = free_pages;
  p.counters = (const long long*)counters;
  p.counters_out = (long long*)counters_out;
  p.first_row = first_row;
  p.status = status_word;
  return launch_tables(p, (cudaStream_t)stream);
}

lava_status lava_page_extend(const lava_cache_desc* cache, const int32_t* add, int32_t max_add,
                             const int32_t* head_rows, int32_t* head_rows_out, int32_t* page_table,
                             int32_t* free_pages, const int64_t* counters, int64_t* counters_out,
                             int32_t* slots, uint32_t* status_word, void* stream) {
  TableParams p = {};
  const lava_status rc = make_cache(cache, &p.c);
  if (rc != LAVA_OK) return rc;
  if (!add || !head_rows || !head_rows_out || !page_table || !free_pages || !counters || !counters_out || !slots)
    return fail(LAVA_ERR_INVALID_ARG, "NULL argument");
  if (max_add < 1) return fail(LAVA_ERR_INVALID_ARG, "max_add must be >= 1");
  p.add = add;
  p.max_add = max_add;
  p.rows = head_rows;
  p.rows_out = head_rows_out;
  p.table = page_table;
  p.ring = free_pages;
  p.ring_out = free_pages;
  p.counters = (const long long*)counters;
  p.counters_out = (long long*)counters_out;
  p.slots = slots;
  p.status = status_word;
  return launch_tables(p, (cudaStream_t)stream);
}

}  // extern "C"
