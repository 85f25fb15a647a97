// Bounds of the keys of a page (include/fc.h, fc_page_bounds): the least and the largest of every dimension of a key head.
//
// A minimum and a maximum need nothing but the keys that are new and what the page's bounds were before, so a step reads no key twice.  A wave
// takes a page and key head at a time: 16 bytes a lane, the lanes of a key side by side, several keys in an instruction and four instructions under way;
// the lanes that hold other keys of the same elements then compare theirs.  Pages with new keys, times heads, of all requests are one row, of which every
// wave has an equal share: a step appends a key to each request or a prompt to a few, and either is spread over the device.
//
// Reading the new keys once bounds it where they are many: 40 prompts, 65536 keys of 8 heads of 128 in pages of 32 (bf16, 143 MB) 29.7 us, 4.8 TB/s; the launch and a
// chain of reads (lengths, page, keys and what was there) where they are not: 64 requests with a key each (bf16) and 37 prompts of 9999 keys,
// 3 heads of 80 (f32, 10 MB), 5.6 us.
#include "operators.hpp"

#include <algorithm>

namespace fc {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

struct BoundsArgs {
  const char *k;
  const int *table, *before, *lengths;
  char *bounds;
  long long k_page, k_place, k_head, b_page, b_head, b_half, table_stride;
  unsigned requests, heads, dim, page, pages, width, workers;
  int lanes;                               // log2 of the lanes of a key
};

// Positions [begin, end) of a request's new keys, and the pages [first, first + count) of its table that hold them
struct NewKeys {
  unsigned begin, end, first, count;
};
__device__ __forceinline__ NewKeys new_keys(const BoundsArgs &a, unsigned b) {
  NewKeys n;
  n.begin = (unsigned)max(a.before[b], 0);
  n.end = (unsigned)min((unsigned long long)max(a.lengths[b], 0), (unsigned long long)a.width * a.page);
  n.first = n.begin / a.page;
  n.count = n.end > n.begin ? (n.end - 1) / a.page - n.first + 1 : 0u;
  return n;
}

template <class T, int N> struct Bounds {
  float low[N], high[N];
  // a NaN stays one
  __device__ __forceinline__ void add(Vec<T, N> x) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      low[i] = __builtin_elementwise_minimum(low[i], (float)x[i]);
      high[i] = __builtin_elementwise_maximum(high[i], (float)x[i]);
    }
  }
};

template <class T> __global__ __launch_bounds__(kThreads) void bounds_kernel(BoundsArgs a) {
  constexpr int N = 16 / sizeof(T), kTogether = 4;
  __shared__ unsigned ends[kThreads];      // of the pages of a thread's requests, summed up to it
  __shared__ unsigned sums[kWaves];
  const unsigned each = (a.requests + kThreads - 1) / kThreads;
  {
    const unsigned b0 = min(threadIdx.x * each, a.requests), b1 = min(b0 + each, a.requests);
    unsigned mine = 0;
    for (unsigned b = b0; b < b1; ++b) mine += new_keys(a, b).count;
    const unsigned upto = (unsigned)wave_scan_inclusive<AddI32>((int)mine);
    if (lane_id() == kWave - 1) sums[wave_id()] = upto;
    __syncthreads();
    unsigned before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (w < wave_id()) before += sums[w];
    ends[threadIdx.x] = before + upto;
    __syncthreads();
  }
  const unsigned total = ends[kThreads - 1], all = total * a.heads, waves = a.workers * kWaves;
  const unsigned share = (all + waves - 1) / waves, wave = blockIdx.x * kWaves + (unsigned)wave_id();
  unsigned at = (unsigned)min((unsigned long long)wave * share, (unsigned long long)all);
  const unsigned end = min(at + share, all);
  const unsigned lanes = 1u << a.lanes, lane = lane_id() & (lanes - 1), key0 = lane_id() >> a.lanes, step = kWave >> a.lanes;
  const unsigned d = lane * N;
  while (at < end) {
    // the request of page `at / heads`
    const unsigned page0 = at / a.heads;
    unsigned chunk = 0;
#pragma unroll
    for (int k = 0; k < kThreads / kWave; ++k) chunk += (unsigned)__popcll(__ballot(ends[k * kWave + lane_id()] <= page0));
    unsigned request = chunk * each, before = chunk ? ends[chunk - 1] : 0u;
    for (;;) {
      const unsigned count = new_keys(a, request).count;
      if (page0 < before + count) break;
      before += count;
      ++request;
    }
    const NewKeys n = new_keys(a, request);
    const unsigned last = min(end, (before + n.count) * a.heads);
    for (; at < last; ++at) {
      const unsigned index = at / a.heads, head = at - index * a.heads, w = n.first + (index - before);
      const unsigned page = (unsigned)a.table[request * a.table_stride + w];
      if (page >= a.pages) continue;
      const unsigned long long start = (unsigned long long)w * a.page;
      const unsigned from = n.begin > start ? n.begin - (unsigned)start : 0u, to = (unsigned)min((unsigned long long)a.page, n.end - start);
      T *const low = reinterpret_cast<T *>(a.bounds) + page * a.b_page + head * a.b_head, *const high = low + a.b_half;
      const T *const keys = reinterpret_cast<const T *>(a.k) + page * a.k_page + head * a.k_head + d;
      Bounds<T, N> x;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x.low[i] = __builtin_inff();
        x.high[i] = -__builtin_inff();
      }
      if (d < a.dim) {
        if (from > 0 && key0 == 0) {       // keys before the new ones
          const Vec<T, N> l = load_vec<T, N>(low + d), h = load_vec<T, N>(high + d);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            x.low[i] = (float)l[i];
            x.high[i] = (float)h[i];
          }
        }
        for (unsigned j = from + key0; j < to; j += kTogether * step) {
          Vec<T, N> v[kTogether];
#pragma unroll
          for (int t = 0; t < kTogether; ++t) v[t] = load_vec<T, N, true>(keys + min(j + t * step, to - 1) * a.k_place);
#pragma unroll
          for (int t = 0; t < kTogether; ++t) x.add(v[t]);
        }
      }
      for (unsigned s = lanes; s < (unsigned)kWave; s *= 2)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          x.low[i] = __builtin_elementwise_minimum(x.low[i], __shfl_xor(x.low[i], (int)s));
          x.high[i] = __builtin_elementwise_maximum(x.high[i], __shfl_xor(x.high[i], (int)s));
        }
      if (d < a.dim && key0 == 0) {
        Vec<T, N> l, h;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          l[i] = (T)x.low[i];
          h[i] = (T)x.high[i];
        }
        store_vec<T, N>(low + d, l);
        store_vec<T, N>(high + d, h);
      }
    }
  }
}

struct PageBounds final : Operator {
  BoundsArgs a{};
  int32_t dtype;
  void record(Recorder &r) const override {
    if (a.requests == 0 || a.heads == 0 || a.pages == 0 || a.width == 0) return;
    if (dtype == FC_F32) r.launch(&bounds_kernel<float>, a.workers, kThreads, a);
    else if (dtype == FC_F16) r.launch(&bounds_kernel<_Float16>, a.workers, kThreads, a);
    else r.launch(&bounds_kernel<__bf16>, a.workers, kThreads, a);
  }
  const char *name() const override { return "page bounds"; }
};

}  // namespace

int make_page_bounds(const fc_page_bounds &n, std::unique_ptr<Operator> &out, std::string &err) {
  TensorChecks c(err);
  const int32_t dtype = n.k_cache.dtype;
  if (dtype != FC_F32 && dtype != FC_F16 && dtype != FC_BF16) return c.fail(FC_E_ARG, "k_cache: type f32, f16 or bf16 is needed").code();
  c.array("k_cache", n.k_cache, dtype, {-1, -1, -1, -1});
  const int64_t pages = n.k_cache.shape[0], page = n.k_cache.shape[1], kv = n.k_cache.shape[2], dim = n.k_cache.shape[3];
  c.array("table", n.table, FC_I32, {-1, -1});
  const int64_t requests = n.table.shape[0], width = n.table.shape[1];
  c.array("lengths_before", n.lengths_before, FC_I32, {requests});
  c.array("lengths", n.lengths, FC_I32, {requests});
  c.array("bounds", n.bounds, dtype, {pages, kv, 2, dim}, true);
  if (!c.ok()) return c.code();
  if (page < 1) return c.fail(FC_E_ARG, "k_cache: pages without places").code();
  if (dim < 8 || dim % 8 || dim > 256) return c.fail(FC_E_UNSUPPORTED, "heads have a multiple of 8 elements, at most 256").code();
  for (const fc_tensor *t : {&n.k_cache, &n.bounds})
    if (pages && kv && common_alignment(*t, 16 / size_of_dtype(dtype)) * size_of_dtype(dtype) != 16)
      return c.fail(FC_E_UNBOUND, "the rows of the cache and of the bounds must be 16-byte aligned").code();
  // pages with new keys, a key head at a time
  uint64_t most;
  const uint64_t of_request = std::min<uint64_t>(width, (0x7fffffffu + (uint64_t)page - 1) / page);
  if (__builtin_mul_overflow(of_request, (uint64_t)requests, &most) || __builtin_mul_overflow(most, (uint64_t)kv, &most) || most > 0x7fffffff)
    return c.fail(FC_E_LIMIT, "too many requests, pages of a request and heads together").code();
  auto op = std::make_unique<PageBounds>();
  op->dtype = dtype;
  BoundsArgs &a = op->a;
  a.k = static_cast<const char *>(n.k_cache.ptr);
  a.table = static_cast<const int *>(n.table.ptr);
  a.before = static_cast<const int *>(n.lengths_before.ptr);
  a.lengths = static_cast<const int *>(n.lengths.ptr);
  a.bounds = static_cast<char *>(n.bounds.ptr);
  a.k_page = n.k_cache.stride[0];
  a.k_place = n.k_cache.stride[1];
  a.k_head = n.k_cache.stride[2];
  a.b_page = n.bounds.stride[0];
  a.b_head = n.bounds.stride[1];
  a.b_half = n.bounds.stride[2];
  a.table_stride = n.table.stride[0];
  a.requests = (unsigned)requests;
  a.heads = (unsigned)kv;
  a.dim = (unsigned)dim;
  a.page = (unsigned)page;
  a.pages = (unsigned)pages;
  a.width = (unsigned)width;
  const unsigned chunks = (unsigned)(dim * size_of_dtype(dtype) / 16);
  while ((1u << a.lanes) < chunks) ++a.lanes;
  const unsigned resident = dtype == FC_F32 ? resident_workgroups(&bounds_kernel<float>, kThreads)
                            : dtype == FC_F16 ? resident_workgroups(&bounds_kernel<_Float16>, kThreads) : resident_workgroups(&bounds_kernel<__bf16>, kThreads);
  a.workers = std::max(1u, std::min(resident ? resident : 2048u, ceil_div(most, kWaves)));
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
