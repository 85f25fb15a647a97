// The pages of a request that count most for a key head (include/fc.h, fc_page_select).
//
// No key of a page scores more with q than  s = sum over d of max(q_d, 0) high_d + min(q_d, 0) low_d,  which is a matrix product: bounds of 16 pages
// are its rows, the query heads of a group its columns.  Its sums are of 64 bits, as is the matrix instruction: which of two pages is taken must not
// depend on the order in which they were added up.  Of the s of a group's heads the largest counts.
//
// The scores become whole numbers of 64 bits in the same order; the k-th largest is found from its upper digits down, 8 bits at a time, from
// the first that differs between the least and the largest on, until the pages above and at it are as many as are wanted.  One workgroup does it
// for a request and key head; where these are few and their pages many, other workgroups help with the scores, and the last to be done selects.
#include "operators.hpp"

#include <algorithm>

namespace fc {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kColumns = 16;
constexpr unsigned long long kAlways = ~0ull;                // above every score; 0, below every score, is a page that is not there

struct SelectArgs {
  const char *q, *bounds;
  const int *table, *lengths;
  int *selected, *selected_lengths;
  unsigned long long *keys;                // DEVICE: of each row `width`; NULL: they fit LDS
  unsigned *counters;                      // DEVICE: one a row, 0 between launches
  long long q_request, q_head, b_page, b_head, b_half, table_stride, s_request, s_head, l_request;
  unsigned requests, heads, group, dim, page, pages, width, most, first, last, parts;
};

using Acc64 = Vec<double, 4>;

// a number that orders scores as they are; NaN counts as infinite, -0 as 0
__device__ __forceinline__ unsigned long long key_of(double s) {
  s = s != s ? __builtin_inf() : s + 0.0;
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, s);
  return bits >> 63 ? ~bits : bits | 1ull << 63;
}

// the largest over the 16 lanes of a row
__device__ __forceinline__ double row_max(double v) {
#pragma unroll
  for (int s = 1; s < 16; s *= 2) v = fmax(v, __shfl_xor(v, s));
  return v;
}

// Scores of the 16 kTiles pages from `at` on of the row's `count`, use(position, key).
template <class T, int Tiles, class Use>
__device__ __forceinline__ void score(const SelectArgs &a, const T *q, const T *bounds, const int *table, unsigned at, unsigned count, Use &&use) {
  constexpr int N = 16 / sizeof(T);
  const unsigned r = lane_id() & 15, g = lane_id() >> 4;
  const T *low[Tiles];
  bool there[Tiles];
#pragma unroll
  for (int t = 0; t < Tiles; ++t) {
    const unsigned w = at + 16 * t + r;
    const unsigned page = w < count ? (unsigned)table[w] : a.pages;
    there[t] = page < a.pages;
    low[t] = bounds + (there[t] ? page * a.b_page : 0ll);
  }
  double best[Tiles][4];
#pragma unroll
  for (int t = 0; t < Tiles; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) best[t][i] = -__builtin_inf();
  for (unsigned head0 = 0; head0 < a.group; head0 += kColumns) {
    Acc64 sums[Tiles];
#pragma unroll
    for (int t = 0; t < Tiles; ++t) sums[t] = Acc64{0.0, 0.0, 0.0, 0.0};
    const bool mine = head0 + r < a.group;
    const T *const from = q + (mine ? (head0 + r) * a.q_head : 0ll);
    for (unsigned d0 = 0; d0 < a.dim; d0 += 4 * N) {
      const unsigned d = d0 + g * N;
      const bool inside = d < a.dim;
      Vec<T, N> x, l[Tiles], h[Tiles];
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = (T)0.0f;
      if (mine && inside) x = load_vec<T, N>(from + d);
#pragma unroll
      for (int t = 0; t < Tiles; ++t) {
#pragma unroll
        for (int e = 0; e < N; ++e) l[t][e] = h[t][e] = (T)0.0f;
        if (there[t] && inside) {
          l[t] = load_vec<T, N>(low[t] + d);
          h[t] = load_vec<T, N>(low[t] + a.b_half + d);
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = (float)x[e];
        // a NaN goes into both
        const double up = (double)(v < 0.0f ? 0.0f : v), down = (double)(v > 0.0f ? 0.0f : v);
#pragma unroll
        for (int t = 0; t < Tiles; ++t) {
          sums[t] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(float)h[t][e], up, sums[t], 0, 0, 0);
          sums[t] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(float)l[t][e], down, sums[t], 0, 0, 0);
        }
      }
    }
    if (mine)
#pragma unroll
      for (int t = 0; t < Tiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) best[t][i] = fmax(best[t][i], sums[t][i] != sums[t][i] ? __builtin_inf() : sums[t][i]);
  }
  // row i of the product's four in this lane: page 4 i + g
#pragma unroll
  for (int t = 0; t < Tiles; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double s = row_max(best[t][i]);
      const unsigned w = at + 16 * t + 4 * i + g;
      const bool is_there = __shfl((int)there[t], 4 * i + (int)g) != 0;
      if (r == 0 && w < count) use(w, !is_there ? 0ull : w < a.first || w + a.last >= count ? kAlways : key_of(s));
    }
}

// Adds this workgroup to `counter`, once what it has stored has arrived; true for the last of `all`.
__device__ __forceinline__ bool last_to_arrive(unsigned *counter, unsigned all) {
  __shared__ unsigned before;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == all - 1) store_agent(counter, 0u);
  }
  __syncthreads();
  return before == all - 1;
}

// The sum over the workgroup up to this thread; total comes back too.  `lds`: kWaves words.
__device__ __forceinline__ unsigned sum_up_to(unsigned v, unsigned *lds, unsigned &total) {
  const unsigned upto = (unsigned)wave_scan_inclusive<AddI32>((int)v);
  __syncthreads();
  if (lane_id() == kWave - 1) lds[wave_id()] = upto;
  __syncthreads();
  unsigned before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave_id()) before += lds[w];
    total += lds[w];
  }
  return before + upto;
}

// Kept: keys in LDS
template <class T, int Kept> __global__ __launch_bounds__(kThreads) void select_kernel(SelectArgs a) {
  constexpr int kTiles = 4;
  __shared__ unsigned long long kept[Kept];
  __shared__ unsigned counts[256], sums[kWaves], found[2];
  __shared__ unsigned long long ends[2][kWaves];
  const unsigned row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
  const unsigned b = row / a.heads, head = row - b * a.heads;
  const unsigned keys = (unsigned)min((unsigned long long)max(load_scalar(a.lengths + b), 0), (unsigned long long)a.width * a.page);
  const unsigned count = (keys + a.page - 1) / a.page;
  const int *const table = a.table + b * a.table_stride;
  int *const selected = a.selected + b * a.s_request + head * a.s_head;
  unsigned long long *const far = a.keys ? a.keys + (size_t)row * a.width : nullptr;
  const bool near = a.parts == 1 && count <= (unsigned)Kept;                   // the keys never leave LDS
  {
    const T *const q = reinterpret_cast<const T *>(a.q) + b * a.q_request + head * a.group * a.q_head;
    const T *const bounds = reinterpret_cast<const T *>(a.bounds) + head * a.b_head;
    const unsigned step = 16 * kTiles * kWaves * a.parts;
    for (unsigned at = (part * kWaves + (unsigned)wave_id()) * 16 * kTiles; at < count; at += step)
      score<T, kTiles>(a, q, bounds, table, at, count, [&](unsigned w, unsigned long long key) {
        if (near) kept[w] = key;
        else store_agent64(far + w, key);
      });
  }
  if (a.parts > 1 && !last_to_arrive(a.counters + row, a.parts)) return;
  if (!near) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (unsigned w = threadIdx.x; w < min(count, (unsigned)Kept); w += kThreads) kept[w] = load_agent64(far + w);
  }
  __syncthreads();
  auto key_at = [&](unsigned w) { return w < (unsigned)Kept ? kept[w] : load_agent64(far + w); };

  // the least and the largest score, and how many pages there are
  unsigned long long least = kAlways, largest = 0;
  unsigned mine = 0, always = 0;
  for (unsigned w = threadIdx.x; w < count; w += kThreads) {
    const unsigned long long key = key_at(w);
    mine += key != 0;
    always += key == kAlways;
    if (key != 0 && key != kAlways) {
      least = min(least, key);
      largest = max(largest, key);
    }
  }
  unsigned candidates, wanted;
  sum_up_to(mine, sums, candidates);
  sum_up_to(always, sums, wanted);
  wanted = a.most - min(wanted, a.most);                                       // of those that are not taken anyway
  // taken: keys above `bar` with their lowest `shift` bits cut off, and of those at it the first `level`
  unsigned long long bar = 0;
  unsigned shift = 0, level = ~0u;
  if (candidates > a.most && wanted == 0) bar = ~0ull, level = 0;
  else if (candidates > a.most) {
#pragma unroll
    for (int s = 1; s < kWave; s *= 2) {
      least = min(least, (unsigned long long)__shfl_xor((long long)least, s));
      largest = max(largest, (unsigned long long)__shfl_xor((long long)largest, s));
    }
    if (lane_id() == 0) { ends[0][wave_id()] = least; ends[1][wave_id()] = largest; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { least = min(least, ends[0][w]); largest = max(largest, ends[1][w]); }
    unsigned bits = least == largest ? 0u : 64u - (unsigned)__clzll((long long)(least ^ largest));   // below which keys differ
    bar = bits == 64 ? 0 : largest >> bits;
    shift = bits;
    level = wanted;
    while (shift > 0) {
      const unsigned digit = min(shift, 8u);
      shift -= digit;
      __syncthreads();
      counts[threadIdx.x] = 0;
      __syncthreads();
      for (unsigned w = threadIdx.x; w < count; w += kThreads) {
        const unsigned long long key = key_at(w);
        if (key != 0 && key != kAlways && (shift + digit == 64 ? 0 : key >> (shift + digit)) == bar) atomicAdd(&counts[key >> shift & ((1u << digit) - 1)], 1u);
      }
      __syncthreads();
      // from the largest digit down: the one where `level` is reached
      const unsigned d = 255u - threadIdx.x, here = counts[d];
      unsigned total;
      const unsigned upto = sum_up_to(here, sums, total);
      if (level > upto - here && level <= upto) { found[0] = d; found[1] = upto - here; }
      __syncthreads();
      bar = bar << digit | found[0];
      level -= found[1];
      if (level == counts[found[0]]) break;                                    // all of them are taken
    }
  }
  // in order: each thread has positions of its own, side by side
  const unsigned each = (count + kThreads - 1) / kThreads, w0 = min(threadIdx.x * each, count), w1 = min(w0 + each, count);
  unsigned above = 0, at_bar = 0;
  for (unsigned w = w0; w < w1; ++w) {
    const unsigned long long key = key_at(w);
    if (key == 0) continue;
    const unsigned long long cut = key >> shift;
    above += candidates <= a.most || key == kAlways || cut > bar;
    at_bar += candidates > a.most && key != kAlways && cut == bar;
  }
  unsigned all_above, all_at;
  const unsigned above_to = sum_up_to(above, sums, all_above), at_to = sum_up_to(at_bar, sums, all_at);
  unsigned level_before = at_to - at_bar, slot = above_to - above + min(level_before, level);
  const unsigned taken = min(all_above + min(all_at, level), a.most);
  bool is_last = false;
  for (unsigned w = w0; w < w1; ++w) {
    const unsigned long long key = key_at(w);
    if (key == 0) continue;
    const unsigned long long cut = key >> shift;
    bool take = candidates <= a.most || key == kAlways || cut > bar;
    if (!take && cut == bar) take = level_before++ < level;
    if (take && slot < a.most) {
      selected[slot++] = table[w];
      is_last |= w + 1 == count;
    }
  }
  for (unsigned k = taken + threadIdx.x; k < a.most; k += kThreads) selected[k] = -1;
  const unsigned short_of = __syncthreads_or(is_last) ? count * a.page - keys : 0u;
  if (threadIdx.x == 0) a.selected_lengths[b * a.l_request + head] = (int)(taken * a.page - short_of);
}

constexpr int kFew = 2048, kMany = 8192;

struct PageSelect final : Operator {
  SelectArgs a{};
  int32_t dtype;
  bool many = false;                       // keys: more than kFew a row, or rows in parts
  template <class F> void with_kernel(F &&f) const {
    auto by = [&](auto t) {
      using T = decltype(t);
      f(many ? &select_kernel<T, kMany> : &select_kernel<T, kFew>);
    };
    if (dtype == FC_F32) by(float{});
    else if (dtype == FC_F16) by(_Float16{});
    else by(__bf16{});
  }
  size_t workspace() const override { return many ? (size_t)a.requests * a.heads * a.width * sizeof(unsigned long long) : 0; }
  void record(Recorder &r) const override {
    if (a.requests == 0 || a.heads == 0) return;
    SelectArgs args = a;
    args.keys = many ? reinterpret_cast<unsigned long long *>(r.workspace) : nullptr;
    args.counters = r.counters;
    with_kernel([&](auto kernel) { r.launch(kernel, a.requests * a.heads * a.parts, kThreads, args); });
  }
  const char *name() const override { return "page select"; }
};

}  // namespace

int make_page_select(const fc_page_select &n, std::unique_ptr<Operator> &out, std::string &err) {
  TensorChecks c(err);
  const int32_t dtype = n.q.dtype;
  if (dtype != FC_F32 && dtype != FC_F16 && dtype != FC_BF16) return c.fail(FC_E_ARG, "q: type f32, f16 or bf16 is needed").code();
  c.array("q", n.q, dtype, {-1, -1, -1});
  const int64_t requests = n.q.shape[0], heads = n.q.shape[1], dim = n.q.shape[2];
  c.array("bounds", n.bounds, dtype, {-1, -1, 2, dim});
  const int64_t pages = n.bounds.shape[0], kv = n.bounds.shape[1];
  c.array("table", n.table, FC_I32, {requests, -1});
  c.array("lengths", n.lengths, FC_I32, {requests});
  c.array("selected", n.selected, FC_I32, {requests, kv, -1}, true);
  c.array("selected_lengths", n.selected_lengths, FC_I32, {requests, kv}, true);
  if (!c.ok()) return c.code();
  const int64_t most = n.selected.shape[2], width = n.table.shape[1];
  if (n.page_size < 1) return c.fail(FC_E_ARG, "page_size must be positive").code();
  if (kv < 1 || heads % kv) return c.fail(FC_E_ARG, "the heads of q must be a multiple of those of the bounds").code();
  if (dim < 8 || dim % 8 || dim > 256) return c.fail(FC_E_UNSUPPORTED, "heads have a multiple of 8 elements, at most 256").code();
  if (n.first < 0 || n.last < 0 || (int64_t)n.first + n.last > most) return c.fail(FC_E_ARG, "first and last must be positive and no more than are selected together").code();
  if (most * n.page_size > 0x7fffffff) return c.fail(FC_E_LIMIT, "the selected pages hold more than 2^31-1 keys").code();
  for (const fc_tensor *t : {&n.q, &n.bounds})
    if (requests && pages && heads && common_alignment(*t, 16 / size_of_dtype(dtype)) * size_of_dtype(dtype) != 16)
      return c.fail(FC_E_UNBOUND, "the rows of q and of the bounds must be 16-byte aligned").code();
  if (requests * kv > 0xffffff) return c.fail(FC_E_LIMIT, "too many requests and heads together").code();
  auto op = std::make_unique<PageSelect>();
  op->dtype = dtype;
  SelectArgs &a = op->a;
  a.q = static_cast<const char *>(n.q.ptr);
  a.bounds = static_cast<const char *>(n.bounds.ptr);
  a.table = static_cast<const int *>(n.table.ptr);
  a.lengths = static_cast<const int *>(n.lengths.ptr);
  a.selected = static_cast<int *>(n.selected.ptr);
  a.selected_lengths = static_cast<int *>(n.selected_lengths.ptr);
  a.q_request = n.q.stride[0];
  a.q_head = n.q.stride[1];
  a.b_page = n.bounds.stride[0];
  a.b_head = n.bounds.stride[1];
  a.b_half = n.bounds.stride[2];
  a.table_stride = n.table.stride[0];
  a.s_request = n.selected.stride[0];
  a.s_head = n.selected.stride[1];
  a.l_request = n.selected_lengths.stride[0];
  a.requests = (unsigned)requests;
  a.heads = (unsigned)kv;
  a.group = (unsigned)(heads / kv);
  a.dim = (unsigned)dim;
  a.page = (unsigned)n.page_size;
  a.pages = (unsigned)pages;
  a.most = (unsigned)most;
  a.first = (unsigned)n.first;
  a.last = (unsigned)n.last;
  // no more than the pages of a request of 2^31-1 keys are looked at
  a.width = (unsigned)std::min<uint64_t>(width, (0x7fffffffu + (uint64_t)a.page - 1) / a.page);
  const unsigned rows = a.requests * a.heads;
  a.parts = rows ? std::max(1u, std::min(1024u / rows, ceil_div(a.width, 64 * kWaves))) : 1u;
  op->many = a.width > (unsigned)kFew || a.parts > 1;
  if ((uint64_t)rows * a.width > (uint64_t)1 << 36) return c.fail(FC_E_LIMIT, "too many requests, heads and pages of a request together").code();
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
