// Attention of drafted tokens over a cache in pages.
//
// Row i of sequence b attends to the len[b] cached tokens and to the drafted tokens that its mask
// names; softmax statistics and sums in fp32.  A row that sees nothing is 0.
#include "attn_common.h"
#include "device_common.h"
#include "rp_internal.h"

namespace rp {

namespace {

constexpr float kLowest = -3.4028235e38f;

__device__ __forceinline__ int tree_len(const TreeArgs& a, int b) { return min(max(a.len[b], 0), a.table_ld << a.lg); }
__device__ __forceinline__ int tree_nodes(const TreeArgs& a, int b) {
  return a.n_nodes ? min(max(a.n_nodes[b], 0), a.N) : a.N;
}
// Drafted tokens 32 w .. 32 w + 31 that row i sees, of n.
__device__ __forceinline__ uint32_t tree_word(const TreeArgs& a, int b, int i, int w, int n) {
  const int below = i - 32 * w;  // without a mask: tokens 0 .. i
  uint32_t m = a.mask ? a.mask[((int64_t)b * a.N + i) * a.W + w] : below < 0 ? 0u : below >= 31 ? ~0u : (2u << below) - 1;
  const int there = n - 32 * w;
  return there >= 32 ? m : there <= 0 ? 0u : m & ((1u << there) - 1);
}

}  // namespace

// One workgroup a (row, head): 256 keys at a time, a thread a key for the scores and a dimension of
// every (256 / D)-th key for the values.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_tree_attn(TreeArgs a) {
  __shared__ float qs[D], p[256], red[16], os[256];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % a.Hq, g = h / (a.Hq / a.Hkv);
  const int row = blockIdx.x / a.Hq, b = row / a.N, i = row % a.N;
  const int nn = tree_nodes(a, b), n0 = tree_len(a, b);
  T* out = (T*)a.out + ((int64_t)row * a.Hq + h) * D;
  if (i >= nn) {
    if (a.zero_rest && tid < D) stf(out + tid, 0.f);
    return;
  }
  if (tid < D) qs[tid] = ldf((const T*)a.q + (int64_t)row * a.q_ld + h * D + tid) * a.scale;
  const int64_t ld = (int64_t)a.Hkv * D;
  auto offset = [&](int t) {  // of key t's row
    int id = a.table[(int64_t)b * a.table_ld + (t >> a.lg)];
    id = min(max(id, 0), a.n_pages - 1);
    return (((int64_t)id << a.lg) + (t & ((1 << a.lg) - 1))) * ld + g * D;
  };
  float m = kLowest, l = 0.f, o = 0.f;
  const int d = tid % D, part = tid / D;
  for (int base = 0; base < n0 + nn; base += 256) {
    __syncthreads();
    const int t = base + tid, j = t - n0;
    const bool seen = t < n0 || (j < nn && (tree_word(a, b, i, j >> 5, nn) >> (j & 31) & 1));
    float s = 0.f;
    if (seen) {
      const T* k = t < n0 ? (const T*)a.k + offset(t) : (const T*)a.kn + ((int64_t)b * a.N + j) * ld + g * D;
      for (int c = 0; c < D; c += 8) {
        float x[8];
        load8(k + c, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], qs[c + e], s);
      }
    }
    float mx = wave_max(seen ? s : -INFINITY);
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float mn = fmaxf(m, mx), alpha = expf(m - mn);
    m = mn;
    const float e = seen ? expf(s - m) : 0.f;
    p[tid] = seen ? e : -1.f;
    l = l * alpha + block_sum(e, red);
    o *= alpha;
    const int cnt = min(256, n0 + nn - base);
    for (int c = part; c < cnt; c += 256 / D) {
      if (p[c] < 0.f) continue;  // a key that is not seen, whatever its value
      const int tk = base + c;
      const T* v = tk < n0 ? (const T*)a.v + offset(tk) : (const T*)a.vn + ((int64_t)b * a.N + tk - n0) * ld + g * D;
      o = fmaf(p[c], ldf(v + d), o);
    }
  }
  os[tid] = o;
  __syncthreads();
  if (tid >= D) return;
  for (int c = 1; c < 256 / D; ++c) o += os[c * D + tid];
  stf(out + tid, l == 0.f ? 0.f : o / l);
}

// One workgroup a sequence, thread i node i: ancestors by walking up.  A parent outside [0, i) is none.
__global__ __launch_bounds__(kMaxNodes) void k_tree_plan(int N, int W, const int32_t* __restrict__ parents,
                                                         const int32_t* __restrict__ pos0, const int32_t* __restrict__ len, int max_pos,
                                                         uint32_t* __restrict__ mask, int32_t* __restrict__ positions) {
  __shared__ int32_t par[kMaxNodes];
  const int b = blockIdx.x, i = threadIdx.x;
  const int64_t row = (int64_t)b * N + i, rows = (int64_t)gridDim.x * N;
  if (i < N) par[i] = parents ? parents[row] : i - 1;
  __syncthreads();
  if (i >= N) return;
  uint32_t words[kMaxNodes / 32] = {};
  int depth = -1;
  for (int at = i, up; at >= 0; at = up) {
#pragma unroll
    for (int w = 0; w < kMaxNodes / 32; ++w)
      if (at >> 5 == w) words[w] |= 1u << (at & 31);
    ++depth;
    up = par[at];
    if (up >= at) up = -1;
  }
#pragma unroll
  for (int w = 0; w < kMaxNodes / 32; ++w)
    if (w < W) mask[row * W + w] = words[w];
  const int64_t p = (int64_t)(pos0 ? pos0[b] : len[b]) + depth;
  const int pos = (int)(p < 0 ? 0 : p >= max_pos ? max_pos - 1 : p);
  positions[row] = pos;
  positions[rows + row] = pos;
  positions[2 * rows + row] = pos;
}

size_t tree_partial_floats(rp_dtype, int32_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_tree_attention(hipStream_t s, rp_dtype dt, const TreeArgs& a) {
  with_storage(dt, [&](auto tag_) {
    using T = decltype(tag_);
    const int grid = a.B * a.N * a.Hq;
    if (a.D == 128)
      k_tree_attn<T, 128><<<grid, 256, 0, s>>>(a);
    else
      k_tree_attn<T, 64><<<grid, 256, 0, s>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_tree_plan(hipStream_t s, int32_t B, int32_t N, int32_t W, const int32_t* parents, const int32_t* pos0,
                            const int32_t* len, int32_t max_pos, uint32_t* mask, int32_t* positions) {
  k_tree_plan<<<B, kMaxNodes, 0, s>>>(N, W, parents, pos0, len, max_pos, mask, positions);
  return hipGetLastError();
}

}  // namespace rp
