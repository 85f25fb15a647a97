// Attention of one new token of each request over its pages of the cache (include/fc.h, fc_paged_attention).
//
// A gather through the block table fused into a fold whose state is (running maximum m, running sum l, weighted sum o):
// a key with score s turns it into (m', l e^(m-m') + e^(s-m'), o e^(m-m') + e^(s-m') v), m' = max(m, s), and two states join the
// same way.
//
// The query heads of a group read the same keys: 16 of them are the columns of the matrix instructions, so a key is read once
// for all of them.  A wave takes 32 keys (16 of 32 bits) at a time and exchanges nothing with other waves until its keys are done:
//   scores  = K q^T     rows: keys,     columns: heads, sum over d;  lane (r, g), r = lane % 16, g = lane / 16, gets those of head r and
//                       the keys 4g .. 4g+3 of every 16
//   outputs = V^T p^T   rows: d,        columns: heads, sum over keys
// The sum over keys takes them in any order, so a lane passes the weights on where the scores left them, and reads the values of
// just these keys, 16 bytes of each at a time, the 16 lanes of a key side by side: rows of V are read in order, and the transposition is
// a permutation of a lane's own registers.
//
// The keys of all requests and key heads are one long row of units of 128 (64) keys, of which every workgroup takes an equal share,
// whatever the lengths are: what is long is split, what is short is taken together.  Pieces of a split row go to scratch; the
// workgroup that is the last of a row to be done joins them in their order, in two steps where they are many.  Where all rows are short and
// they are many, a wave takes one at a time instead, and nothing is exchanged at all.
//
// Reading the cache once bounds it where that is long, the launch and a chain of reads (lengths, page, keys, pieces) where it is not:
//   one request of 131072 keys, 8 key heads of 128, 64 heads (bf16, 537 MB) 85 to 88 us, 6.1 to 6.3 TB/s; 64 requests of 1 to 8192 keys, 254057 together,
//   8 key heads of 128 (bf16, 1041 MB) 179 us, 5.8 TB/s, over pages of 24, 8 or 1 205 us, 5.1 TB/s; 16 requests of 16384 keys, 8 key heads
//   of 256 (bf16, 2147 MB) 313 us, 6.9 TB/s, of 192 253 us, 6.4 TB/s; 37 requests in windows of 1000 keys, 6 key heads of 96, pages of 24 (f32, 111 MB)
//   28 to 30 us, 3.7 to 4.0 TB/s, where the six units of a workgroup are too few to hide its start and end; 4 requests of up to 300 keys,
//   2 key heads of 64 (f16) 7.1 us.
//
// The forms beside that share the kernel's code and differ in where a row's table and length lie and in how it ends.  A table for each key head: the rows of lengths
// are those of requests and key heads; 64 requests, 8 key heads, 64 pages of 32 keys each (bf16, 521 MB) 92 us, 5.7 TB/s; one request of 128 pages a head
// 13 us, the chain of reads.  Behind a prefix: whoever has the whole of a row joins its prefix' pieces as well, eight at a time; 200 requests of 1024 keys on
// average, 4 key heads of 128 behind a prefix of 4096 (bf16, 430 MB and 40 of pieces) 112 to 124 us, 4.2 TB/s; 64 of 500, 8 key heads behind 32768 keys
// (131 MB and 38 of pieces) 50 to 60 us, rows of four units whose ends and joins little else covers.  That form takes no row by a wave, which
// would leave the prefix' pieces to a wave each.
#pragma once

#include "operators.hpp"
#include "prefix.hpp"

namespace fc {

// What a call is: attention over one table a request, over one for each of its key heads, or over what a request has behind the prefix of
// its group, whose pieces are joined with it.
enum class Form { kPlain, kHeads, kAfterPrefix };

struct AttentionArgs {
  const char *q, *k, *v;
  const int *table, *lengths;
  char *out;
  float *lse;                              // NULL: not wanted
  float *pieces;                           // DEVICE: two pieces a workgroup
  unsigned *counters;                      // DEVICE: two a workgroup, 0 between launches
  long long q_request, q_head, out_request, out_head, lse_request, table_stride;
  long long k_page, k_place, k_head, v_page, v_place, v_head;
  unsigned requests, kv_heads, group, tiles, dim, page, pages, width, window;      // tiles: a group's heads, 16 at a time
  unsigned workers, streams;               // workgroups; as many of them as keep the memory busy with long rows
  bool wide_out;                           // rows of out are 16-byte aligned
  unsigned page_factor, page_shift;        // n / (page / 16) = n * page_factor >> page_shift, n below 2^30
  float scale;
  long long table_head, length_request;    // Form::kHeads: between a request's tables, and between the lengths of two requests
  unsigned heads;                          // Form::kHeads: key heads; `requests` are all their rows, `kv_heads` is 1
  const unsigned *prefix_plan;             // Form::kAfterPrefix (prefix.hpp)
  const float *prefix_pieces;
  unsigned prefix_columns;
};

using AttentionKernel = void (*)(AttentionArgs);
// the kernel of a form for this type, these heads and pages (one translation unit for each form)
template <Form F> AttentionKernel attention_kernel_of(int32_t dtype, unsigned dim, bool even);

// An operator that ends in the attention kernel.
struct Attention : Operator {
  AttentionArgs a{};
  int32_t dtype = FC_F32;
  Form form = Form::kPlain;
  bool even = false;
  unsigned most_units = 0;                 // the call can have
  AttentionKernel kernel() const;
  // as many workgroups as the device holds at once, but no more than there can be units
  void settle_workers();
  size_t workspace() const override;
  void record(Recorder &r) const override;
  const char *name() const override { return "paged attention"; }
};
// The arrays that all forms have, checked and entered into `op`, whose form is set.
int settle_attention(const fc_paged_attention &n, Attention &op, std::string &err);

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr unsigned kMostDim = 256;
constexpr unsigned kLongRow = 8;           // units
constexpr unsigned kShortRow = 2;          // units
constexpr int kColumns = 16;               // query heads of a group that are taken together
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;


// A call's row b of lengths, and what its keys belong to.
struct Place {
  unsigned request, kv;                    // kv: its only key head (Form::kHeads), else 0
};
template <Form F> __device__ __forceinline__ Place place_of(const AttentionArgs &a, unsigned b) {
  if constexpr (F != Form::kHeads) return {b, 0u};
  const unsigned request = b / a.heads;
  return {request, b - request * a.heads};
}
template <Form F> __device__ __forceinline__ const int *length_of(const AttentionArgs &a, unsigned b) {
  if constexpr (F != Form::kHeads) return a.lengths + b;
  const Place p = place_of<F>(a, b);
  return a.lengths + p.request * a.length_request + p.kv;
}

template <Form F> __device__ __forceinline__ const int *table_of(const AttentionArgs &a, unsigned b, const Place &p) {
  if constexpr (F != Form::kHeads) return a.table + b * a.table_stride;
  return a.table + p.request * a.table_stride + p.kv * a.table_head;
}

// What the types differ in.  kKeys: keys of a wave's step; kShift: the weights are held 2^kShift larger, which keeps the small ones
// of 16-bit floats off their smallest numbers.
template <class T> struct Kind { static constexpr int kKeys = 32, kShift = 0; };
template <> struct Kind<_Float16> { static constexpr int kKeys = 32, kShift = 14; };
template <> struct Kind<float> { static constexpr int kKeys = 16, kShift = 0; };

template <class T> constexpr int kUnit = Kind<T>::kKeys * kWaves;

using Acc = Vec<float, 4>;
__device__ __forceinline__ Acc mma(Vec<__bf16, 8> a, Vec<__bf16, 8> b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ Acc mma(Vec<_Float16, 8> a, Vec<_Float16, 8> b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ Acc mma(Vec<float, 4> a, Vec<float, 4> b, Acc c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// A weight as two numbers of 16 bits: the upper part cut off, not rounded, so that the rest is not negative, and the rest not 0 where the
// upper part is not, so that an infinite value times a weight stays that infinity in both products.  Together 16 bits (bf16) or 22 of the
// weight, which leaves a result as exact as its own 16 bits hold it; a third part would make the matrix instructions of the values half as
// many again.  A weight below the smallest number, 2^-38 of the largest one for f16, is rounded to it or to 0: it must not add
// up over the keys.  The median is the larger of what is left and the smallest number where the weight is above that, else the weight.
__device__ __forceinline__ void split(float p, __bf16 &high, __bf16 &low) {
  const float cut = __uint_as_float(__float_as_uint(p) & 0xffff0000u);
  high = (__bf16)cut;
  low = (__bf16)__builtin_amdgcn_fmed3f(p - cut, 0x1p-126f, p);
}
__device__ __forceinline__ void split(float p, _Float16 &high, _Float16 &low) {
  high = (_Float16)__builtin_amdgcn_cvt_pkrtz(p, 0.0f)[0];
  low = (_Float16)__builtin_amdgcn_fmed3f(p - (float)high, 0x1p-24f, p);
}

// 2^shift e^x, x not above 0.  The difference from the maximum is taken before it is put into powers of 2, so that the rounding of large scores
// cancels; a scale that is a power of 2 then leaves scores as exact as their products.
__device__ __forceinline__ float exp_of(float x, float shift = 0.0f) { return __builtin_amdgcn_exp2f(fmaf(x, kLog2e, shift)); }

// over the lanes of a head: lane, lane ^ 16, lane ^ 32, lane ^ 48.  Swapping a register's odd rows of 16 lanes with another's even ones,
// or its upper half with the other's lower one, leaves the two values that belong together in the two.
template <class F> __device__ __forceinline__ float over_column(float v, F &&f) {
  auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
  s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float column_max(float v) { return over_column(v, [](float x, float y) { return fmaxf(x, y); }); }
__device__ __forceinline__ float column_sum(float v) { return over_column(v, [](float x, float y) { return x + y; }); }

// a value that all lanes have, in scalar registers
__device__ __forceinline__ unsigned uniform(unsigned v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ unsigned long long uniform(unsigned long long v) { return (unsigned long long)uniform((unsigned)(v >> 32)) << 32 | uniform((unsigned)v); }

// Keys of a request: [begin, end), from the step boundary `from` on in `units` units.
struct Span {
  unsigned begin, end, from, units;
};
template <class T> __device__ __forceinline__ Span span_of(const AttentionArgs &a, int length) {
  Span s;
  s.end = a.pages ? (unsigned)min((unsigned long long)max(length, 0), (unsigned long long)a.width * a.page) : 0u;
  s.begin = a.window && length > 0 && (unsigned)length > a.window ? (unsigned)length - a.window : 0u;
  s.from = s.begin / Kind<T>::kKeys * Kind<T>::kKeys;
  s.units = s.end > s.begin ? (s.end - s.from + kUnit<T> - 1) / kUnit<T> : 0u;
  return s;
}

// This workgroup's share of all units: units [at, end) of the row, the first of them `offset` units into request `request`.
struct Share {
  unsigned at, end, offset, share, request;
  bool by_wave;                            // every row is short, and they are many: a wave takes a row at a time
};

template <Form F, class T> __device__ __forceinline__ Share share_of(const AttentionArgs &a, unsigned worker) {
  __shared__ unsigned sums[kWaves], found_offset, found;     // the top bit of a sum, which is below 2^31: a row is long
  const unsigned rows = a.kv_heads * a.tiles, each = (a.requests + kThreads - 1) / kThreads;
  const unsigned b0 = min(threadIdx.x * each, a.requests), b1 = min(b0 + each, a.requests);
  unsigned mine = 0, most = 0;
  for (unsigned b = b0; b < b1; ++b) {
    const unsigned units = span_of<T>(a, *length_of<F>(a, b)).units;
    mine += units;
    most = max(most, units);
  }
  mine *= rows;
  const unsigned upto = (unsigned)wave_scan_inclusive<AddI32>((int)mine);
  const unsigned is_long = __any(most > kShortRow) ? 0x80000000u : 0u;
  if (lane_id() == kWave - 1) sums[wave_id()] = upto | is_long;
  __syncthreads();
  unsigned before = 0, total = 0, any_long = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const unsigned sum = sums[w] & 0x7fffffffu;
    any_long |= sums[w] ^ sum;
    if (w < wave_id()) before += sum;
    total += sum;
  }
  Share s;
  total = uniform(total);
  // a row costs a workgroup about 6 us from its first page to its result, whatever its length.  Where none is longer than two units and they are
  // more than the workgroups, a wave takes a whole row, which exchanges nothing and hides the others' waits (93 requests of 25 keys, 11 key heads,
  // 192 elements of 16 bits 12 us, 26 by workgroups; 256 of 256 keys, 8 key heads of 128 48 us and 54); longer rows of unequal length
  // would leave waves idle (200 of up to 500 keys 57 us, 51 by workgroups), few rows all but a few (64 of 256 keys 21 us and 16.5)
  s.by_wave = F != Form::kAfterPrefix && uniform(any_long) == 0 && a.requests * rows > a.workers;
  // long rows keep a compute unit's memory pipe full with few workgroups, and the fewer they are the less is joined; short ones leave
  // gaps that others fill: one workgroup a compute unit and all that are resident take for a request of 131072 keys 88 and 102 us, 100 of 1000
  // keys 75 and 84, 200 of up to 1000 89 and 84.5, 200 of up to 500 60 and 51.  Behind a prefix each row ends with the prefix' pieces, which others'
  // keys hide: 200 requests of 1024 keys on average, 4 key heads 128 us and 115
  const unsigned workers = F != Form::kAfterPrefix && total >= kLongRow * a.requests * rows ? a.streams : a.workers;
  s.share = max((total + workers - 1) / workers, 1u);
  s.at = (unsigned)min((unsigned long long)worker * s.share, (unsigned long long)total);
  s.end = min(s.at + s.share, total);
  before += upto - mine;
  if (s.at >= before && s.at < before + mine) {
    unsigned b = b0;
    for (; b + 1 < b1; ++b) {
      const unsigned here = span_of<T>(a, *length_of<F>(a, b)).units * rows;
      if (s.at < before + here) break;
      before += here;
    }
    found = b;
    found_offset = s.at - before;
  }
  __syncthreads();
  s.request = s.at < s.end ? uniform(found) : 0u;
  s.offset = s.at < s.end ? uniform(found_offset) : 0u;
  return s;
}

// floats of a piece: the weighted sums of the heads, then (m, l) of each
__device__ __host__ __forceinline__ unsigned rows_of_piece(unsigned group) { return group < (unsigned)kColumns ? group : (unsigned)kColumns; }
__device__ __host__ __forceinline__ unsigned long long piece_floats(unsigned group, unsigned dim) { return (unsigned long long)rows_of_piece(group) * (dim + 2); }

// Hints of a load: kept, or read once and not worth keeping.  A key's line is read in two instructions, which keeps it; a value's in one, and
// the way past the caches is the faster (64 ragged requests 212 us, 193 this way, 201 with the keys past the caches too).
constexpr int kKept = 0, kStream = 2;

// 16 (or 8) bytes of a lane through a descriptor; zeros where the offset lies past its end
template <int Hint, class T, int N> __device__ __forceinline__ Vec<T, N> load_buffer(__amdgpu_buffer_rsrc_t from, unsigned offset) {
  if constexpr (sizeof(T) * N == 16)
    return __builtin_bit_cast(Vec<T, N>, __builtin_amdgcn_raw_buffer_load_b128(from, (int)offset, 0, Hint));
  else
    return __builtin_bit_cast(Vec<T, N>, __builtin_amdgcn_raw_buffer_load_b64(from, (int)offset, 0, Hint));
}

// One wave's heads, and their state.  Even: every 16 keys from a multiple of 16 on lie on one page, and 16 keys of it span less than
// 2^31 bytes: the page is then the wave's, its descriptor lies in scalar registers, and the lanes' offsets into 16 keys never change;
// what is not there (other requests' keys, elements past D, pages outside the cache) is an offset or a descriptor that gives zeros.
// Otherwise every lane looks its keys up.
template <class T, int Dim, bool Even> struct Wave {
  static constexpr int kKeys = Kind<T>::kKeys, kSub = kKeys / 16, kWide = 16 / sizeof(T);      // kWide: elements of 16 bytes
  static constexpr int kChunks = Dim / (4 * kWide);          // of K: 16 bytes of each of 4 lanes
  static constexpr int kW = Dim / 16;                        // d of a lane in V: parts n of kPart from (16 n + r) kPart on
  static constexpr int kParts = kW < kWide ? 1 : kW / kWide, kPart = kW < kWide ? kW : kWide;  // ... in loads of 16 bytes at most
  static constexpr unsigned kNothing = 0x80000000u;          // beyond every descriptor
  using Frag = Vec<T, kWide>;
  using Part = Vec<T, kPart>;

  // Where the keys of a step lie: the page of each 16 (Even), or of the lane's key of each 16.  a.pages: nowhere.
  struct Where {
    unsigned j0, page[kSub], place[kSub];
  };

  const AttentionArgs &a;
  const Span s;
  const int *table;
  const T *k, *v;
  unsigned r, g, k_at[kChunks], v_at[4][kParts];             // offsets in bytes into 16 keys (Even): of key r, and of keys 4g .. 4g+3
  Frag q[kChunks], kf[kSub][kChunks];
  Part vf[kSub][4][kParts];
  bool there[kSub][4];                                       // the keys 4g + i of vf (not Even)
  Acc o[kW];
  float m, l;

  __device__ __forceinline__ Wave(const AttentionArgs &args, const Span &span, const int *pages, unsigned b, unsigned kv, unsigned head0, unsigned count)
      : a(args), s(span), table(pages), k(reinterpret_cast<const T *>(args.k) + kv * args.k_head),
        v(reinterpret_cast<const T *>(args.v) + kv * args.v_head), r(lane_id() & 15), g(lane_id() >> 4) {
    const T *heads = reinterpret_cast<const T *>(a.q) + b * a.q_request + head0 * a.q_head;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const unsigned d = (c * 4 + g) * kWide;
      Frag f;
#pragma unroll
      for (int i = 0; i < kWide; ++i) f[i] = (T)0.0f;
      if (r < count && d < a.dim) f = load_vec<T, kWide>(heads + r * a.q_head + d);
      q[c] = f;
      if constexpr (Even) k_at[c] = d < a.dim ? (unsigned)(r * a.k_place + d) * sizeof(T) : kNothing;
    }
    if constexpr (Even)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < kParts; ++n)
          v_at[i][n] = (16 * n + r) * kPart < a.dim ? (unsigned)((4 * g + i) * a.v_place + (16 * n + r) * kPart) * sizeof(T) : kNothing;
#pragma unroll
    for (int j = 0; j < kW; ++j) o[j] = Acc{0.0f, 0.0f, 0.0f, 0.0f};
    m = -__builtin_inff();
    l = 0.0f;
  }

  // which d of its head o[j][i] is
  __device__ __forceinline__ unsigned d_of(int i, int j) const { return (j / kPart * 16 + 4 * g + i) * kPart + j % kPart; }

  __device__ __forceinline__ bool inside(unsigned j) const { return j - s.begin < s.end - s.begin; }       // s.end > s.begin

  // Whether there is anything of a head in chunk c.  The last quarter of them is left out where it is not, but only where a chunk is four slow matrix
  // instructions and the pages are of any size: 37 requests of up to 3001 keys, pages of 24 and 7, heads of 40, 48, 72, 96, 160 and 192 elements of
  // 32 bits take 2 to 7 % less so (96 elements 40.6 us, 43.2 without), of 112 1 %, of 128 and 256 the same; 16 bits or even pages lose 2 to 7 %.
  __device__ __forceinline__ bool in_use(int c) const { return sizeof(T) == 2 || Even || c < kChunks * 3 / 4 || (unsigned)(c * 4 * kWide) < a.dim; }

  __device__ __forceinline__ Where locate(unsigned j0) const {
    Where w;
    w.j0 = j0;
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      if constexpr (Even) {
        const unsigned n = min(j0 + 16 * u, s.end - 1) / 16; // past the end: the last 16, whose page is then not looked at
        const unsigned at = (unsigned)((unsigned long long)n * a.page_factor >> a.page_shift);
        const unsigned page = (unsigned)load_scalar(table + at);
        w.page[u] = j0 + 16 * u < s.end ? page : a.pages;
        w.place[u] = 16 * n - at * a.page;
      } else {
        const unsigned j = j0 + 16 * u + r;
        w.page[u] = a.pages;
        w.place[u] = 0;
        if (inside(j)) {
          const unsigned at = j / a.page;
          w.page[u] = (unsigned)table[at];
          w.place[u] = j - at * a.page;
        }
      }
    }
    return w;
  }

  // whether every key of a step is there (Even)
  __device__ __forceinline__ bool all_there(const Where &w) const {
    bool all = w.j0 >= s.begin && w.j0 + kKeys <= s.end;
#pragma unroll
    for (int u = 0; u < kSub; ++u) all &= w.page[u] < a.pages;
    return all;
  }

  // descriptor of 16 keys: it ends behind the last that is there
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t keys_of(const T *cache, long long page_stride, long long place_stride, const Where &w, int u) const {
    const bool there = w.page[u] < a.pages;
    const T *base = cache + (there ? w.page[u] * page_stride + w.place[u] * place_stride : 0ll);
    const unsigned keys = min(s.end - min(w.j0 + 16 * u, s.end), 16u);
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(uniform((unsigned long long)base)), 0,
                                             uniform(there ? keys * (unsigned)place_stride * (unsigned)sizeof(T) : 0u), 0x00027000);
  }

  __device__ __forceinline__ void load_keys(const Where &w) {
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      if constexpr (Even) {
        const auto from = keys_of(k, a.k_page, a.k_place, w, u);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) kf[u][c] = load_buffer<kKept, T, kWide>(from, k_at[c]);
      } else {
        // what is not there reads a place that is, and is put right where it is used: nothing has to wait here
        const bool mine = w.page[u] < a.pages;
        const T *row = k + (mine ? w.page[u] * a.k_page + w.place[u] * a.k_place : 0ll);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          const unsigned d = (c * 4 + g) * kWide;
          if (in_use(c)) kf[u][c] = load_vec<T, kWide>(row + (d < a.dim ? d : 0u));
        }
      }
    }
  }

  __device__ __forceinline__ void load_values(const Where &w) {
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      if constexpr (Even) {
        const auto from = keys_of(v, a.v_page, a.v_place, w, u);
        // keys before the window give zeros: a weight of zero would not do where they are not finite
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int n = 0; n < kParts; ++n) vf[u][i][n] = load_buffer<kStream, T, kPart>(from, w.j0 + 16 * u + 4 * g + i < s.begin ? kNothing : v_at[i][n]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned page = __shfl(w.page[u], (int)(4 * g + i)), place = __shfl(w.place[u], (int)(4 * g + i));
          const bool mine = page < a.pages;
          there[u][i] = mine;
          const T *row = v + (mine ? page * a.v_page + place * a.v_place : 0ll);
#pragma unroll
          for (int n = 0; n < kParts; ++n) vf[u][i][n] = load_vec<T, kPart>(row + ((16 * n + r) * kPart < a.dim ? (16 * n + r) * kPart : 0u));
        }
      }
    }
  }

  // Zeros for what load_keys and load_values read in place of what is not there (not Even): keys past D of a head, whose query is zero
  // there, and the values of keys that have none, whose weight is, would be more than nothing where they are not finite.  Elements
  // past D of the values make sums that nobody reads.
  __device__ __forceinline__ void clear_keys() {
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if ((c * 4 + 4) * kWide > (int)a.dim)
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
          for (int i = 0; i < kWide; ++i) kf[u][c][i] = (c * 4 + g) * kWide < a.dim ? kf[u][c][i] : (T)0.0f;
  }
  __device__ __forceinline__ void clear_values() {
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < kParts; ++n)
#pragma unroll
          for (int e = 0; e < kPart; ++e) vf[u][i][n][e] = there[u][i] ? vf[u][i][n][e] : (T)0.0f;
  }

  // weights of the keys of `w` from kf, the state brought up to them
  __device__ __forceinline__ void weigh(const Where &w, float (&p)[kSub][4]) {
    bool all = Even && all_there(w);
    if constexpr (!Even) {
      clear_keys();
      bool mine = true;
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine &= there[u][i];
      all = __all(mine);
      if (!all) clear_values();
    }
    float most = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      // in four sums where products are of 32 bits: the rounding of one long sum is most of the result's error, and four halve it
      constexpr int kSums = sizeof(T) == 4 ? 4 : 1;
      Acc part[kSums];
#pragma unroll
      for (int c = 0; c < kSums; ++c) part[c] = Acc{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
        if (in_use(c)) part[c % kSums] = mma(kf[u][c], q[c], part[c % kSums]);
      Acc score = part[0];
      if constexpr (kSums == 4) score = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) p[u][i] = score[i] * a.scale;
    }
    if (!all) {
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool mine = Even ? w.page[u] < a.pages && inside(w.j0 + 16 * u + 4 * g + i) : there[u][i];
          if (!mine) p[u][i] = -__builtin_inff();
        }
    }
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, p[u][i]);
    most = fmaxf(column_max(most), m);
    const float top = most == -__builtin_inff() ? 0.0f : most;
    if (__any(most > m)) {                                   // of any head: the maxima settle after a few keys
      const float keep = exp_of(m - top);
      m = most;
      l *= keep;
#pragma unroll
      for (int j = 0; j < kW; ++j) o[j] *= keep;
    }
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[u][i] = exp_of(p[u][i] - top, (float)Kind<T>::kShift);
        l += p[u][i];
      }
  }

  // the sums of vf with the weights
  __device__ __forceinline__ void sum(const float (&p)[kSub][4]) {
    if constexpr (sizeof(T) == 2) {
      Vec<T, 8> high, low;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        T upper, rest;
        split(p[e / 4][e % 4], upper, rest);
        high[e] = upper;
        low[e] = rest;
      }
#pragma unroll
      for (int n = 0; n < kParts; ++n) {
        const Part v0 = vf[0][0][n], v1 = vf[0][1][n], v2 = vf[0][2][n], v3 = vf[0][3][n], v4 = vf[1][0][n], v5 = vf[1][1][n], v6 = vf[1][2][n], v7 = vf[1][3][n];
#pragma unroll
        for (int e = 0; e < kPart; ++e) {
          const Vec<T, 8> values = {v0[e], v1[e], v2[e], v3[e], v4[e], v5[e], v6[e], v7[e]};
          Acc &sums = o[n * kPart + e];
          sums = mma(values, high, sums);
          sums = mma(values, low, sums);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < kW; ++j)
        o[j] = mma(Vec<float, 4>{vf[0][0][j / kPart][j % kPart], vf[0][1][j / kPart][j % kPart], vf[0][2][j / kPart][j % kPart], vf[0][3][j / kPart][j % kPart]},
                   Vec<float, 4>{p[0][0], p[0][1], p[0][2], p[0][3]}, o[j]);
    }
  }

  // The steps at j0, j0 + step, .. below `end`.  The keys of the next step are asked for once this one's are used up, its values likewise,
  // and the pages two steps ahead: steps past the end ask for nothing.
  __device__ __forceinline__ void run(unsigned j0, unsigned end, unsigned step) {
    if (j0 >= end) return;
    Where now = locate(j0), next = locate(j0 + step);
    load_keys(now);
    load_values(now);
    for (;;) {
      Where after = locate(next.j0 + step);
      float p[kSub][4];
      weigh(now, p);
      const bool more = next.j0 < end;
      if (more) load_keys(next);
      sum(p);
      if (!more) break;
      load_values(next);
      now = next;
      next = after;
    }
  }
};

// log sum of a row; the logarithm is the instruction's (1 ulp) of a sum that is never below 2^kShift
template <class T> __device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? -__builtin_inff() : m + (__log2f(l) - (float)Kind<T>::kShift) * kLn2;
}

// A row that one wave has done: its lanes write what they hold.
template <class W, class T> __device__ __forceinline__ void write_wave(const AttentionArgs &a, const W &w, unsigned b, unsigned head0, unsigned count, float l, T *) {
  if (w.r >= count) return;
  const unsigned head = head0 + w.r;
  T *to = reinterpret_cast<T *>(a.out) + b * a.out_request + head * a.out_head;
  const float by_l = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int j = 0; j < W::kW; j += W::kPart)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned d = w.d_of(i, j);
      if (d >= a.dim) continue;
      typename W::Part x;
#pragma unroll
      for (int e = 0; e < W::kPart; ++e) x[e] = (T)(w.o[j + e][i] * by_l);
      if (a.wide_out) store_vec<T, W::kPart, false>(to + d, x);
      else
#pragma unroll
        for (int e = 0; e < W::kPart; ++e) to[d + e] = x[e];
    }
  if (a.lse && w.g == 0) a.lse[b * a.lse_request + head] = log_sum<T>(w.m, l);
}

// What a request's keys behind the prefix of its group left, joined with the prefix' pieces of this head (Form::kAfterPrefix).
__device__ __forceinline__ void join_prefix(const AttentionArgs &a, unsigned b, unsigned head, unsigned d, Vec<float, 4> &sum, float &m, float &l) {
  constexpr unsigned kTogether = 8;
  const PrefixPlan plan(a.prefix_plan);
  const PrefixOf of = plan.of(b);
  if (of.units == 0) return;
  const unsigned kv = head / a.group, column = of.index * a.group + (head - kv * a.group);
  const unsigned block = column / a.prefix_columns, row = kv * of.blocks + block, at = column - block * a.prefix_columns;
  const unsigned start = of.start + row * of.units, share = plan.share();
  const unsigned w0 = start / share, n = (start + of.units - 1) / share - w0 + 1;
  const unsigned long long first = (unsigned long long)w0 + of.row + row;
  const size_t piece = prefix_piece_floats(a.prefix_columns, a.dim);
  for (unsigned p = 0; p < n; p += kTogether) {
    Vec<float, 4> x[kTogether];
    Vec<float, 2> e[kTogether];
#pragma unroll
    for (unsigned k = 0; k < kTogether; ++k) {
      const float *from = a.prefix_pieces + (first + min(p + k, n - 1)) * piece;
      x[k] = load_vec<float, 4>(from + (size_t)at * a.dim + d);
      e[k] = load_vec<float, 2>(from + (size_t)a.prefix_columns * a.dim + 2 * at);
      if (p + k >= n) e[k] = Vec<float, 2>{-__builtin_inff(), 0.0f};
    }
    float most = m;
#pragma unroll
    for (unsigned k = 0; k < kTogether; ++k) most = fmaxf(most, e[k][0]);
    const float base = most == -__builtin_inff() ? 0.0f : most, keep = exp_of(m - base);
    m = most;
    l *= keep;
    sum *= keep;
#pragma unroll
    for (unsigned k = 0; k < kTogether; ++k) {
      const float f = exp_of(e[k][0] - base);
      l += e[k][1] * f;
      if (p + k < n) sum += x[k] * f;
    }
  }
}

template <Form F, class T> __device__ __forceinline__ void write_result(const AttentionArgs &a, unsigned b, unsigned head, unsigned d, Vec<float, 4> sum, float m, float l) {
  if constexpr (F == Form::kAfterPrefix) join_prefix(a, b, head, d, sum, m, l);
  Vec<T, 4> x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (T)(l == 0.0f ? 0.0f : sum[i] / l);
  T *to = reinterpret_cast<T *>(a.out) + b * a.out_request + head * a.out_head + d;
#pragma unroll
  for (int i = 0; i < 4; ++i) to[i] = x[i];
  if (a.lse && d == 0) a.lse[b * a.lse_request + head] = log_sum<T>(m, l);
}

// A piece: the weighted sums of the heads, then (m, l) of each.  It is written and read around the caches that compute units do not
// share, two floats at a time: fences that write these caches back and empty them would do it for all that passes through
// them (a launch of one long request 323 us, this way 122).
struct Piece {
  unsigned long long *sums, *ends;
  __device__ __forceinline__ Piece(const AttentionArgs &a, unsigned long long slot)
      : sums(reinterpret_cast<unsigned long long *>(a.pieces + slot * piece_floats(a.group, a.dim))), ends(sums + rows_of_piece(a.group) * a.dim / 2) {}
  static __device__ __forceinline__ unsigned long long pair(float x, float y) { return (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x); }
  static __device__ __forceinline__ Vec<float, 2> pair(unsigned long long w) { return {__uint_as_float((unsigned)w), __uint_as_float((unsigned)(w >> 32))}; }
  __device__ __forceinline__ void store(unsigned at, Vec<float, 4> x) const {
    store_agent64(sums + at / 2, pair(x[0], x[1]));
    store_agent64(sums + at / 2 + 1, pair(x[2], x[3]));
  }
  __device__ __forceinline__ Vec<float, 4> load(unsigned at) const {
    const Vec<float, 2> x = pair(load_agent64(sums + at / 2)), y = pair(load_agent64(sums + at / 2 + 1));
    return {x[0], x[1], y[0], y[1]};
  }
  __device__ __forceinline__ void store_end(unsigned head, float m, float l) const { store_agent64(ends + head, pair(m, l)); }
  __device__ __forceinline__ Vec<float, 2> load_end(unsigned head) const { return pair(load_agent64(ends + head)); }
};

// The pieces of a split row, made by the workers w0 .. w1 whose shares it reaches into.  The first is its worker's last piece where the
// row starts inside of a share; all others are their workers' first.
struct SplitRow {
  unsigned w0, w1, group, groups;          // joined `group` at a time, counted from the end
  bool starts_inside;
  __device__ __forceinline__ SplitRow(const Share &s, unsigned start, unsigned end) {
    w0 = start / s.share;
    w1 = (end - 1) / s.share;
    starts_inside = start != w0 * s.share;
    const unsigned n = w1 - w0 + 1;
    group = n <= 16 ? n : (unsigned)ceilf(sqrtf((float)n));
    groups = (n + group - 1) / group;
  }
  __device__ __forceinline__ unsigned long long slot(unsigned w) const { return w * 2ull + (w == w0 && starts_inside); }
  __device__ __forceinline__ unsigned last_of_group(unsigned k) const { return w1 - k * group; }
  __device__ __forceinline__ unsigned first_of_group(unsigned k) const { return max((int)w0, (int)(w1 - k * group - group) + 1); }
};

// Adds this workgroup to `counter`, once what its waves have stored has arrived; true for the last of `all`, who may then read
// what the others stored before.
__device__ __forceinline__ bool last_to_arrive(unsigned *counter, unsigned all) {
  __shared__ unsigned before;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == all - 1) store_agent(counter, 0u);
  }
  __syncthreads();
  const bool last = before == all - 1;
  __syncthreads();
  return last;
}

// The pieces slot(0) .. slot(n - 1), of `count` heads, as one: use(head, d, sum, m, l) for four d at a time.
template <class Slot, class Use> __device__ __forceinline__ void join(const AttentionArgs &a, unsigned n, unsigned count, Slot &&slot, Use &&use) {
  constexpr int kTogether = 8;
  const unsigned quads = a.dim / 4;
  for (unsigned i = threadIdx.x; i < count * quads; i += kThreads) {
    const unsigned head = i / quads, d = i % quads * 4;
    float m = -__builtin_inff(), l = 0.0f;
    Vec<float, 4> sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (unsigned p = 0; p < n; p += kTogether) {
      Vec<float, 4> x[kTogether];
      Vec<float, 2> e[kTogether];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const Piece piece(a, slot(min(p + k, n - 1)));
        x[k] = piece.load(head * a.dim + d);
        e[k] = piece.load_end(head);
        if (p + k >= n) e[k] = Vec<float, 2>{-__builtin_inff(), 0.0f};
      }
      float most = m;
#pragma unroll
      for (int k = 0; k < kTogether; ++k) most = fmaxf(most, e[k][0]);
      const float base = most == -__builtin_inff() ? 0.0f : most, keep = exp_of(m - base);
      m = most;
      l *= keep;
      sum *= keep;
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const float f = exp_of(e[k][0] - base);
        l += e[k][1] * f;
        if (p + k < n) sum += x[k] * f;
      }
    }
    use(head, d, sum, m, l);
  }
}

// A kernel keeps 80 to 239 of its scalars (arguments, strides, descriptors) in lanes of vector registers, the more the larger its heads, and no vector
// register in memory; heads of more than 128 elements take more than 256 registers, so that a SIMD has one wave.
template <Form F, class T, int Dim, bool Even>
__global__ __launch_bounds__(kThreads, Dim == 256 ? 1 : Dim == 128 ? (Even && sizeof(T) == 2 ? 3 : 2) : Even ? 4 : 3) void attention_kernel(AttentionArgs a) {
  __shared__ float sums[kWaves][kColumns][Dim + 4];          // + 4: the heads' rows start at different banks
  __shared__ float tops[kWaves][kColumns], totals[kWaves][kColumns];
  const unsigned rows = a.kv_heads * a.tiles, worker = blockIdx.x;
  const unsigned r = lane_id() & 15, g = lane_id() >> 4;
  for (unsigned b = worker; b < a.requests; b += a.workers) {          // requests without a key
    if (span_of<T>(a, load_scalar(length_of<F>(a, b))).units) continue;
    const Place place = place_of<F>(a, b);
    for (unsigned i = threadIdx.x; i < a.kv_heads * a.group * (a.dim / 4); i += kThreads)
      write_result<F, T>(a, place.request, place.kv * a.group + i / (a.dim / 4), i % (a.dim / 4) * 4, Vec<float, 4>{0.0f, 0.0f, 0.0f, 0.0f}, F == Form::kAfterPrefix ? -__builtin_inff() : 0.0f, 0.0f);
  }
  Share s = share_of<F, T>(a, worker);
  if (__builtin_expect(s.by_wave, 0)) {
    for (unsigned turn = worker * kWaves + uniform((unsigned)wave_id()); turn < a.requests * rows; turn += a.workers * kWaves) {
      const unsigned b = turn / rows, row = turn - b * rows;
      const Span span = span_of<T>(a, load_scalar(length_of<F>(a, b)));
      if (span.units == 0) continue;
      const Place place = place_of<F>(a, b);
      const unsigned kv = place.kv + row / a.tiles, head0 = kv * a.group + row % a.tiles * kColumns;
      const unsigned count = min((unsigned)kColumns, (kv + 1) * a.group - head0);
      Wave<T, Dim, Even> w(a, span, table_of<F>(a, b, place), place.request, kv, head0, count);
      w.run(span.from, span.end, Kind<T>::kKeys);
      write_wave(a, w, place.request, head0, count, column_sum(w.l), (T *)nullptr);
    }
    return;
  }
  const unsigned share_begin = s.at;
  while (s.at < s.end) {
    const unsigned b = s.request;
    const Span span = span_of<T>(a, load_scalar(length_of<F>(a, b)));
    if (s.offset >= span.units * rows) { s.offset -= span.units * rows; ++s.request; continue; }
    const unsigned row = s.offset / span.units, unit0 = s.offset - row * span.units, unit1 = min(span.units, unit0 + (s.end - s.at));
    const Place place = place_of<F>(a, b);
    const unsigned kv = place.kv + row / a.tiles, head0 = kv * a.group + row % a.tiles * kColumns;
    const unsigned count = min((unsigned)kColumns, (kv + 1) * a.group - head0);
    Wave<T, Dim, Even> w(a, span, table_of<F>(a, b, place), place.request, kv, head0, count);
    w.run(span.from + unit0 * kUnit<T> + uniform((unsigned)wave_id()) * Kind<T>::kKeys, min(span.end, span.from + unit1 * kUnit<T>), kUnit<T>);
    const float total = column_sum(w.l);
    __syncthreads();                                         // the row before is read
    if (g == 0) { tops[wave_id()][r] = w.m; totals[wave_id()][r] = total; }
    if (r < count)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < Dim / 16; j += 4) {
          Vec<float, 4> x = {w.o[j][i], w.o[j + 1][i], w.o[j + 2][i], w.o[j + 3][i]};
          *reinterpret_cast<Vec<float, 4> *>(&sums[wave_id()][r][w.d_of(i, j)]) = x;
        }
    __syncthreads();
    const bool whole = unit0 == 0 && unit1 == span.units;
    const Piece mine(a, worker * 2ull + (s.at != share_begin));
    for (unsigned i = threadIdx.x; i < count * (Dim / 4); i += kThreads) {
      const unsigned head = i / (Dim / 4), d = i % (Dim / 4) * 4;
      if (d >= a.dim) continue;
      float most = tops[0][head], sum_l = 0.0f;
#pragma unroll
      for (int n = 1; n < kWaves; ++n) most = fmaxf(most, tops[n][head]);
      Vec<float, 4> x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < kWaves; ++n) {
        const float f = most == -__builtin_inff() ? 0.0f : exp_of(tops[n][head] - most);
        sum_l += totals[n][head] * f;
        x += *reinterpret_cast<const Vec<float, 4> *>(&sums[n][head][d]) * f;
      }
      if (whole) write_result<F, T>(a, place.request, head0 + head, d, x, most, sum_l);
      else {
        mine.store(head * a.dim + d, x);
        if (d == 0) mine.store_end(head, most, sum_l);
      }
    }
    if (!whole) {
      const SplitRow split(s, s.at - unit0, s.at - unit0 + span.units);
      const unsigned k = (split.w1 - worker) / split.group, last = split.last_of_group(k), of_group = last - split.first_of_group(k) + 1;
      // a group of one has nothing to join, and no counter: a worker's counter belongs to the row that ends in its share, or covers it
      bool joins = of_group == 1 || last_to_arrive(a.counters + last, of_group);
      if (joins && split.groups > 1) {
        if (of_group > 1) {
          const Piece to(a, split.slot(last));
          join(a, of_group, count, [&](unsigned p) { return split.slot(last - p); }, [&](unsigned head, unsigned d, Vec<float, 4> sum, float m, float l) {
            to.store(head * a.dim + d, sum);                 // only this thread reads these four
            if (d == 0) { tops[0][head] = m; totals[0][head] = l; }
          });
          __syncthreads();                                   // all have read the ends that are written over
          if (threadIdx.x < count) to.store_end(threadIdx.x, tops[0][threadIdx.x], totals[0][threadIdx.x]);
        }
        joins = last_to_arrive(a.counters + a.workers + split.w1, split.groups);
      }
      if (joins)
        join(a, split.groups > 1 ? split.groups : of_group, count, [&](unsigned p) { return split.slot(split.groups > 1 ? split.last_of_group(p) : last - p); },
             [&](unsigned head, unsigned d, Vec<float, 4> sum, float m, float l) { write_result<F, T>(a, place.request, head0 + head, d, sum, m, l); });
    }
    s.at += unit1 - unit0;
    s.offset += unit1 - unit0;
  }
}


template <Form F, class T> AttentionKernel attention_kernel_of_type(unsigned dim, bool even) {
  if (dim <= 64) return even ? &attention_kernel<F, T, 64, true> : &attention_kernel<F, T, 64, false>;
  if (dim <= 128) return even ? &attention_kernel<F, T, 128, true> : &attention_kernel<F, T, 128, false>;
  return even ? &attention_kernel<F, T, 256, true> : &attention_kernel<F, T, 256, false>;
}

}  // namespace

template <Form F> AttentionKernel attention_kernel_of(int32_t dtype, unsigned dim, bool even) {
  if (dtype == FC_F32) return attention_kernel_of_type<F, float>(dim, even);
  if (dtype == FC_F16) return attention_kernel_of_type<F, _Float16>(dim, even);
  return attention_kernel_of_type<F, __bf16>(dim, even);
}

}  // namespace fc
