// Attention of one new token over the pages of a paged cache.
//
// One block per (query head, layer and sequence), tiles of 1024 rows, fp32 throughout: logits in the base-2
// domain, running maximum and sum, then the product with V.  Rows are read with 16-byte loads, d / 4 or d / 8
// lanes per row.
#include <algorithm>

#include <math.h>

#include "sm100_ptx.cuh"

namespace lava {
namespace {

using namespace sm100;

constexpr int kThreads = 256;
constexpr int kTile = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PageParams {
  Cache c;
  int first_layer;
  const void* q;           // [layers, batch, H_q, d]
  const char* k_pages;
  const char* v_pages;
  const int* table;
  const int* rows;
  void* out;
  float* lse;
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads)
decode_pages_kernel(const PageParams p) {
  in_stream_order();
  constexpr int kPer = BF16 ? 8 : 4;  // elements per 16-byte load
  constexpr int kLanes = D / kPer;    // lanes per row
  constexpr int kGroups = kThreads / kLanes;
  __shared__ float pr[kTile], red[8];
  __shared__ float sums[kGroups][D];
  const Cache& c = p.c;
  const int h = blockIdx.x, prob = blockIdx.y;
  const size_t head = ((size_t)p.first_layer * c.batch + prob) * c.n_kv_heads + h / c.group;
  const int len = (int)min((long long)max(0, p.rows[head]), (long long)c.max_pages << c.page_shift);
  const int* pages = p.table + head * c.max_pages;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = tid / kLanes, col = tid % kLanes;
  auto unpack = [](const uint4& raw, float (&x)[kPer]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (BF16) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      } else {
        x[j] = __uint_as_float(w[j]);
      }
    }
  };
  auto row_piece = [&](const char* pool, int row) {  // zeros where the page is none of the pool
    const int page = pages[row >> c.page_shift];
    if ((unsigned)page >= (unsigned)c.n_pages) return uint4{};
    const long long at = ((long long)page << c.page_shift) + (row & (c.page_rows - 1));
    return reinterpret_cast<const uint4*>(pool)[at * kLanes + col];
  };
  auto block_reduce = [&](float x, auto op) {  // the same order in every thread
    for (int o = 16; o > 0; o >>= 1) x = op(x, __shfl_xor_sync(0xffffffffu, x, o));
    __syncthreads();
    if (lane == 0) red[warp] = x;
    __syncthreads();
    x = red[0];
    for (int w = 1; w < kThreads / 32; ++w) x = op(x, red[w]);
    return x;
  };
  float q[kPer];
  unpack(reinterpret_cast<const uint4*>(p.q)[((long long)prob * c.n_q_heads + h) * kLanes + col], q);
  float m = -INFINITY, l = 0.f, acc[kPer] = {};
  for (int i0 = 0; i0 < len; i0 += kTile) {
    const int cnt = min(kTile, len - i0);
    float best = -INFINITY;
    for (int r0 = 0; r0 < cnt; r0 += kGroups) {
      const int r = r0 + group;
      float x[kPer], z = 0.f;
      unpack(r < cnt ? row_piece(p.k_pages, i0 + r) : uint4{}, x);
#pragma unroll
      for (int j = 0; j < kPer; ++j) z = fmaf(q[j], x[j], z);
      for (int o = kLanes / 2; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
      z *= c.scale;
      if (c.softcap > 0.f) z = c.softcap * tanhf(z / c.softcap);
      z *= kLog2e;
      if (r < cnt) {
        best = fmaxf(best, z);
        if (col == 0) pr[r] = z;
      }
    }
    const float m_new = fmaxf(m, block_reduce(best, [](float a, float b) { return fmaxf(a, b); }));
    float sum = 0.f;
    for (int r = tid; r < cnt; r += kThreads) {
      const float e = exp2f(pr[r] - m_new);
      pr[r] = e;
      sum += e;
    }
    sum = block_reduce(sum, [](float a, float b) { return a + b; });  // also: all of pr is written
    const float corr = exp2f(m - m_new);
    l = l * corr + sum;
#pragma unroll
    for (int j = 0; j < kPer; ++j) acc[j] *= corr;
    m = m_new;
    for (int r = group; r < cnt; r += kGroups) {
      float x[kPer];
      unpack(row_piece(p.v_pages, i0 + r), x);
#pragma unroll
      for (int j = 0; j < kPer; ++j) acc[j] = fmaf(pr[r], x[j], acc[j]);
    }
    __syncthreads();  // pr is written again
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) sums[group][col * kPer + j] = acc[j];
  __syncthreads();
  const size_t at = (size_t)prob * c.n_q_heads + h;
  if (tid < D) {
    float x = 0.f;
    for (int i = 0; i < kGroups; ++i) x += sums[i][tid];
    x = len > 0 ? x / l : 0.f;
    if constexpr (BF16)
      reinterpret_cast<__nv_bfloat16*>(p.out)[at * D + tid] = __float2bfloat16_rn(x);
    else
      reinterpret_cast<float*>(p.out)[at * D + tid] = x;
  }
  if (p.lse && tid == 0) p.lse[at] = len > 0 ? (m + log2f(l)) * kLn2 : -INFINITY;
}

constexpr size_t kStatusBytes = 256;

}  // namespace
}  // namespace lava

using namespace lava;

extern "C" {

size_t lava_cache_workspace_bytes(const lava_cache_desc* cache) {
  Cache c;
  return make_cache(cache, &c) == LAVA_OK ? kStatusBytes : 0;
}

lava_status lava_decode_attention_pages(const lava_cache_desc* cache, int32_t first_layer, int32_t n_layers,
                                        const void* q, const void* k_pages, const void* v_pages,
                                        const int32_t* page_table, const int32_t* head_rows, void* out, float* lse,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  PageParams p;
  const lava_status rc = make_cache(cache, &p.c);
  if (rc != LAVA_OK) return rc;
  const Cache& c = p.c;
  if (n_layers < 1 || first_layer < 0 || first_layer > c.n_layers - n_layers)
    return fail(LAVA_ERR_INVALID_ARG, "layers %d ... %lld are not all in a cache of %d", first_layer,
                (long long)first_layer + n_layers - 1, c.n_layers);
  if (!q || !k_pages || !v_pages || !page_table || !head_rows || !out)
    return fail(LAVA_ERR_INVALID_ARG, "NULL argument");
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out))
    return fail(LAVA_ERR_INVALID_ARG, "q, k_pages, v_pages and out must be 16-byte aligned");
  if ((long long)n_layers * c.batch > 65535)
    return fail(LAVA_ERR_UNSUPPORTED, "n_layers*batch must be <= 65535");
  const size_t need = lava_cache_workspace_bytes(cache);
  if (!workspace || workspace_bytes < need)
    return fail(LAVA_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
  if (!aligned16(workspace)) return fail(LAVA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  p.first_layer = first_layer;
  p.q = q;
  p.k_pages = (const char*)k_pages;
  p.v_pages = (const char*)v_pages;
  p.table = page_table;
  p.rows = head_rows;
  p.out = out;
  p.lse = lse;
  const auto kernel = c.dtype == LAVA_BF16
                          ? (c.head_dim == 64 ? decode_pages_kernel<64, true> : decode_pages_kernel<128, true>)
                          : (c.head_dim == 64 ? decode_pages_kernel<64, false> : decode_pages_kernel<128, false>);
  const cudaError_t e = launch_in_order(kernel, dim3(c.n_q_heads, n_layers * c.batch), kThreads, 0,
                                        (cudaStream_t)stream, p);
  count_launches(1);
  return check_cuda(e, "paged decode attention launch");
}

}  // extern "C"
