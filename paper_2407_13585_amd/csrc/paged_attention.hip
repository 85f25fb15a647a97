// Attention of one new token of each request over its pages of the cache (include/fc.h, fc_paged_attention).
//
// A gather through the block table fused into a fold whose state is (running maximum m, running sum l, weighted sum o):
// a key with score s turns it into (m', l e^(m-m') + e^(s-m'), o e^(m-m') + e^(s-m') v), m' = max(m, s), and two states join the
// same way.  A workgroup takes one query head of one request; its waves take 64 keys in turn and join at the end.
#include "operators.hpp"

#include <cmath>

namespace fc {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr unsigned kMostDim = 256;

struct AttentionArgs {
  const char *q, *k, *v;
  const int *table, *lengths;
  char *out;
  float *lse;                       // NULL: not wanted
  long long q_request, q_head, out_request, out_head, lse_request, table_stride;
  long long k_page, k_place, k_head, v_page, v_place, v_head;
  unsigned heads, group, dim, page, pages, width, window;
  float scale;
};

template <class T>
__global__ __launch_bounds__(kThreads) void attention_kernel(AttentionArgs a) {
  __shared__ float query[kMostDim], weights[kWaves][kWave], sums[kWaves][kMostDim], tops[kWaves], totals[kWaves];
  const unsigned b = blockIdx.y, h = blockIdx.x, kv = h / a.group;
  const T *q = reinterpret_cast<const T *>(a.q) + b * a.q_request + h * a.q_head;
  for (unsigned d = threadIdx.x; d < a.dim; d += kThreads) query[d] = (float)q[d] * a.scale;
  __syncthreads();
  const int length = max(a.lengths[b], 0);
  const unsigned begin = a.window && (unsigned)length > a.window ? (unsigned)length - a.window : 0u;
  const unsigned end = (unsigned)min((unsigned long long)length, (unsigned long long)a.width * a.page);
  const int *table = a.table + b * a.table_stride;
  float top = -__builtin_inff(), total = 0.0f, o[kMostDim / kWave] = {};
  for (unsigned j0 = begin + wave_id() * kWave; j0 < end; j0 += kThreads) {
    const unsigned j = j0 + lane_id();
    const unsigned page = j < end ? (unsigned)table[j / a.page] : a.pages;
    float s = -__builtin_inff();
    if (page < a.pages) {
      const T *k = reinterpret_cast<const T *>(a.k) + page * a.k_page + j % a.page * a.k_place + kv * a.k_head;
      s = 0.0f;
      for (unsigned d = 0; d < a.dim; d += 8) {
        const Vec<T, 8> x = load_vec<T, 8>(k + d);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(query[d + i], (float)x[i], s);
      }
    }
    float most = s;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    most = fmaxf(most, top);
    const float base = most == -__builtin_inff() ? 0.0f : most;
    const float p = page < a.pages ? expf(s - base) : 0.0f, keep = expf(top - base);
    float sum = p;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    total = total * keep + sum;
    top = most;
    weights[wave_id()][lane_id()] = p;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < (int)(kMostDim / kWave); ++i) o[i] *= keep;
    for (unsigned n = 0; n < (unsigned)kWave; ++n) {
      const unsigned at = __shfl(page, (int)n), jn = j0 + n;
      if (at >= a.pages) continue;
      const float weight = weights[wave_id()][n];
      const T *v = reinterpret_cast<const T *>(a.v) + at * a.v_page + jn % a.page * a.v_place + kv * a.v_head;
#pragma unroll
      for (int i = 0; i < (int)(kMostDim / kWave); ++i)
        if (i * kWave + lane_id() < (int)a.dim) o[i] = fmaf(weight, (float)v[i * kWave + lane_id()], o[i]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  if (lane_id() == 0) { tops[wave_id()] = top; totals[wave_id()] = total; }
#pragma unroll
  for (int i = 0; i < (int)(kMostDim / kWave); ++i) sums[wave_id()][i * kWave + lane_id()] = o[i];
  __syncthreads();
  float most = tops[0];
  for (int w = 1; w < kWaves; ++w) most = fmaxf(most, tops[w]);
  const float base = most == -__builtin_inff() ? 0.0f : most;
  float l = 0.0f;
  for (int w = 0; w < kWaves; ++w) l += totals[w] * expf(tops[w] - base);
  for (unsigned d = threadIdx.x; d < a.dim; d += kThreads) {
    float x = 0.0f;
    for (int w = 0; w < kWaves; ++w) x += sums[w][d] * expf(tops[w] - base);
    reinterpret_cast<T *>(a.out)[b * a.out_request + h * a.out_head + d] = (T)(l == 0.0f ? 0.0f : x / l);
  }
  if (a.lse && threadIdx.x == 0) a.lse[b * a.lse_request + h] = l == 0.0f ? -__builtin_inff() : base + logf(l);
}

struct PagedAttention final : Operator {
  AttentionArgs a{};
  int32_t dtype;
  unsigned requests;
  void record(Recorder &r) const override {
    if (requests == 0 || a.heads == 0) return;
    auto go = [&](auto element) { r.launch(&attention_kernel<decltype(element)>, a.heads, kThreads, a); r.launches.back().grid.y = requests; };
    if (dtype == FC_F32) go(float{});
    else if (dtype == FC_F16) go(_Float16{});
    else go(__bf16{});
  }
  const char *name() const override { return "paged attention"; }
};

}  // namespace

int make_paged_attention(const fc_paged_attention &n, std::unique_ptr<Operator> &out, std::string &err) {
  TensorChecks c(err);
  const int32_t dtype = n.q.dtype;
  if (dtype != FC_F32 && dtype != FC_F16 && dtype != FC_BF16) return c.fail(FC_E_ARG, "q: type f32, f16 or bf16 is needed").code();
  c.array("q", n.q, dtype, {-1, -1, -1});
  const int64_t requests = n.q.shape[0], heads = n.q.shape[1], dim = n.q.shape[2];
  c.array("k_cache", n.k_cache, dtype, {-1, -1, -1, dim});
  const int64_t pages = n.k_cache.shape[0], page = n.k_cache.shape[1], kv = n.k_cache.shape[2];
  c.array("v_cache", n.v_cache, dtype, {pages, page, kv, dim});
  c.array("table", n.table, FC_I32, {requests, -1});
  c.array("lengths", n.lengths, FC_I32, {requests});
  c.array("out", n.out, dtype, {requests, heads, dim}, true);
  if (present(n.lse)) c.array("lse", n.lse, FC_F32, {requests, heads}, true);
  if (!c.ok()) return c.code();
  if (page < 1) return c.fail(FC_E_ARG, "k_cache: pages without places").code();
  if (kv < 1 || heads % kv) return c.fail(FC_E_ARG, "the heads of q must be a multiple of those of the cache").code();
  if (dim < 8 || dim % 8 || dim > (int64_t)kMostDim) return c.fail(FC_E_UNSUPPORTED, "heads have a multiple of 8 elements, at most 256").code();
  if (!std::isfinite(n.scale)) return c.fail(FC_E_ARG, "scale must be finite").code();
  if (n.window < 0) return c.fail(FC_E_ARG, "window must not be negative").code();
  if (requests > 65535) return c.fail(FC_E_LIMIT, "more than 65535 requests").code();
  for (const fc_tensor *t : {&n.k_cache, &n.v_cache})
    if (pages && common_alignment(*t, 16 / size_of_dtype(dtype)) * size_of_dtype(dtype) != 16) return c.fail(FC_E_UNBOUND, "the caches' rows must be 16-byte aligned").code();
  auto op = std::make_unique<PagedAttention>();
  op->dtype = dtype;
  op->requests = (unsigned)requests;
  AttentionArgs &a = op->a;
  a.q = static_cast<const char *>(n.q.ptr);
  a.k = static_cast<const char *>(n.k_cache.ptr);
  a.v = static_cast<const char *>(n.v_cache.ptr);
  a.table = static_cast<const int *>(n.table.ptr);
  a.lengths = static_cast<const int *>(n.lengths.ptr);
  a.out = static_cast<char *>(n.out.ptr);
  a.lse = present(n.lse) ? static_cast<float *>(n.lse.ptr) : nullptr;
  a.q_request = n.q.stride[0];
  a.q_head = n.q.stride[1];
  a.out_request = n.out.stride[0];
  a.out_head = n.out.stride[1];
  a.lse_request = n.lse.stride[0];
  a.table_stride = n.table.stride[0];
  a.k_page = n.k_cache.stride[0];
  a.k_place = n.k_cache.stride[1];
  a.k_head = n.k_cache.stride[2];
  a.v_page = n.v_cache.stride[0];
  a.v_place = n.v_cache.stride[1];
  a.v_head = n.v_cache.stride[2];
  a.heads = (unsigned)heads;
  a.group = (unsigned)(heads / kv);
  a.dim = (unsigned)dim;
  a.page = (unsigned)page;
  a.pages = (unsigned)pages;
  a.width = (unsigned)n.table.shape[1];
  a.window = (unsigned)n.window;
  a.scale = (float)n.scale;
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
