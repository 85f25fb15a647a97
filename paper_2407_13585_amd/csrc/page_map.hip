// Block tables and slot maps of one step of a server (include/fc.h, fc_page_map).
//
// Three prefix sums over the requests (new tokens, pages taken, pages given back), then every thread finds the request of the first of
// four tokens by bisection in the first of them, and with it positions and pages: a scan, two gathers and two scatters, and nothing
// between them but the sums.  The bytes are few (16 a token, 20 a request), so a step costs its launches and the chain of dependent
// reads of one token.  Up to 4096 requests every workgroup sums all of them for itself and keeps the sums in LDS, which makes a
// step one launch (1024 threads a workgroup; 256 up to 1024 requests, whose barriers and scans are shorter); above, two kernels
// leave the sums in scratch for the third.  What there is of each request is written by a workgroup of its own.
//   64 requests, a token each: 5.5 to 6.1 us (the launch is about 3.5 of it); 1000 requests, 60013 tokens (1.2 MB): 6.9 us (7.6 with 1024 threads a workgroup);
//   4096 requests, 2^20 tokens (17 MB): 11.5 us, 1.5 TB/s (17.8 with a token a thread): the sums, a search in LDS, a page and a store one behind another,
//   588 vector instructions a wave, many of them divisions by the page size; a token each 8.3 us, of 4097 requests in three launches 21.5 us;
//   65536 requests, 2^20 tokens 29.5 us.
#include "operators.hpp"

namespace fc {

namespace {

constexpr int kPerThread = 4;                      // requests of a thread, and tokens
constexpr unsigned kRequestsOfGroup = 32;          // pages given back ask for workgroups too: a step of 2231 requests, half of which leave, 9.8 us, 10.8 without
constexpr int kMany = 1024, kFew = 256;            // threads of a workgroup
constexpr int kChunk = kMany * kPerThread;         // requests that a workgroup of many threads sums at once

struct PageMapArgs {
  const int *lengths, *fresh;
  int *pool;
  const long long *cursor;
  int *table;
  int *lengths_after, *row_start;
  long long *slots;
  int *positions, *request;
  long long *cursor_after, *unplaced;
  long long table_stride;
  unsigned requests, width, page, tokens, entries;
  bool wide;                                       // the arrays of an entry a request, or a token, begin at 16 bytes
};

// At most the entries of the table, which are below 2^31, and tokens, whose sums stay at 2^32-1 where they would pass it.
struct Sums {
  unsigned tokens, taken, given;
};
struct AddTokens {
  using T = unsigned;
  static __device__ __forceinline__ T identity() { return 0u; }
  static __device__ __forceinline__ T apply(T a, T b) { return __builtin_elementwise_add_sat(a, b); }
};
__device__ __forceinline__ Sums operator+(Sums a, Sums b) { return {AddTokens::apply(a.tokens, b.tokens), a.taken + b.taken, a.given + b.given}; }

struct Request {
  int length, fresh;
  unsigned want, have, goal;                       // want: below 2^32, the sum of two values below 2^31
  __device__ __forceinline__ Sums sums() const { return {fresh > 0 ? (unsigned)fresh : 0u, goal > have ? goal - have : 0u, have > goal ? have - goal : 0u}; }
};

__device__ __forceinline__ unsigned pages_of(const PageMapArgs &a, unsigned n) {
  const unsigned q = n / a.page;
  return min(q + (n != q * a.page ? 1u : 0u), a.width);
}

__device__ __forceinline__ Request request_of(const PageMapArgs &a, int length, int fresh) {
  Request q;
  q.length = max(length, 0);
  q.fresh = fresh;
  const long long want = (long long)q.length + q.fresh;
  q.want = want > 0 ? (unsigned)want : 0u;
  q.have = pages_of(a, (unsigned)q.length);
  q.goal = pages_of(a, q.want);
  return q;
}
__device__ __forceinline__ Request request_at(const PageMapArgs &a, unsigned r) { return request_of(a, a.lengths[r], a.fresh[r]); }

// The ring of free pages, at places counted from the cursor's own.
struct Ring {
  unsigned head, tail, available;
  __device__ __forceinline__ Ring(const PageMapArgs &a) {
    const long long h = a.cursor[0], t = a.cursor[1], n = a.entries;
    available = (unsigned)min(max(t - h, 0ll), n);
    head = place_of(h, n);
    tail = place_of(t, n);
  }
  static __device__ __forceinline__ unsigned place_of(long long at, long long n) {
    if (n == 0) return 0u;
    if ((unsigned long long)at >> 32 == 0) return (unsigned)at % (unsigned)n;        // as long as the ring has not turned that often
    return (unsigned)((at % n + n) % n);
  }
  // `k` below the number of entries
  static __device__ __forceinline__ unsigned place(const PageMapArgs &a, unsigned from, unsigned k) {
    const unsigned p = from + k;                   // both below 2^31
    return p >= a.entries ? p - a.entries : p;
  }
  __device__ __forceinline__ unsigned got(unsigned first, unsigned taken) const { return first < available ? min(available - first, taken) : 0u; }
};

__device__ __forceinline__ unsigned stored_tokens(const PageMapArgs &a, const Request &q, unsigned got) {
  const unsigned long long room = (unsigned long long)(q.fresh > 0 ? q.have + got : a.width) * a.page;
  return (unsigned)min((unsigned long long)q.want, room);
}

__device__ __forceinline__ Sums sums_of_lane(Sums v, int lane) {
  return {(unsigned)__builtin_amdgcn_readlane((int)v.tokens, lane), (unsigned)__builtin_amdgcn_readlane((int)v.taken, lane),
          (unsigned)__builtin_amdgcn_readlane((int)v.given, lane)};
}

// Sums of the threads before this one; total: of all.  lds: an entry a wave, free when the call returns.
template <int Threads> __device__ __forceinline__ Sums block_scan_exclusive(Sums v, Sums *lds, Sums &total) {
  const Sums upto = {wave_scan_inclusive<AddTokens>(v.tokens), (unsigned)wave_scan_inclusive<AddI32>((int)v.taken), (unsigned)wave_scan_inclusive<AddI32>((int)v.given)};
  __syncthreads();
  if (lane_id() == kWave - 1) lds[wave_id()] = upto;
  __syncthreads();
  // every wave sums the waves' sums again: at most 16, a lane each
  static_assert(Threads / kWave <= 16, "one row of lanes");
  const Sums of_wave = lds[lane_id() & (Threads / kWave - 1)];
  const Sums waves = {row_scan_inclusive<AddTokens>(of_wave.tokens), (unsigned)row_scan_inclusive<AddI32>((int)of_wave.taken),
                      (unsigned)row_scan_inclusive<AddI32>((int)of_wave.given)};
  __syncthreads();
  total = sums_of_lane(waves, Threads / kWave - 1);
  const Sums before = wave_id() ? sums_of_lane(waves, __builtin_amdgcn_readfirstlane(wave_id()) - 1) : Sums{0, 0, 0};
  // of the lanes before this one: its own value cannot be taken away again where the sum of the tokens stopped
  const Sums lanes = {lane_prev(0u, upto.tokens), lane_prev(0u, upto.taken), lane_prev(0u, upto.given)};
  return before + lanes;
}

template <int Threads> __device__ __forceinline__ long long block_sum(long long v, long long *lds) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
  __syncthreads();
  if (lane_id() == 0) lds[wave_id()] = v;
  __syncthreads();
  long long sum = 0;
#pragma unroll
  for (int w = 0; w < Threads / kWave; ++w) sum += lds[w];
  return sum;
}

__device__ __forceinline__ unsigned token_of(unsigned sum) { return min(sum, 0x7fffffffu); }

using Four = Vec<unsigned, kPerThread>;

// Of each request: the tokens, taken and given pages of those before it, and its own length; padded to whole chunks.
struct Starts {
  unsigned *row, *first, *behind, *length;
};

// The sums before each request of [begin, begin + Threads * kPerThread), what comes before them added; the arrays of one entry a
// request are written too where `writes`.  Returns the sums up to the end, and the thread's unplaced tokens.
template <int Threads>
__device__ __forceinline__ Sums scan_chunk(const PageMapArgs &a, const Ring &ring, unsigned begin, Sums before, Starts to, bool writes, Sums *lds, long long &unplaced) {
  Request q[kPerThread];
  Sums mine = {0, 0, 0};
  const unsigned r0 = begin + threadIdx.x * kPerThread;
  if (a.wide && r0 + kPerThread <= a.requests) {
    const auto length = *reinterpret_cast<const Vec<int, kPerThread> *>(a.lengths + r0), fresh = *reinterpret_cast<const Vec<int, kPerThread> *>(a.fresh + r0);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) q[k] = request_of(a, length[k], fresh[k]);
  } else {
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) q[k] = r0 + k < a.requests ? request_at(a, r0 + k) : request_of(a, 0, 0);
  }
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) mine = mine + q[k].sums();
  Sums total;
  Sums s = before + block_scan_exclusive<Threads>(mine, lds, total);
  unplaced = 0;
  Four row, first, behind, length;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    row[k] = token_of(s.tokens);
    first[k] = s.taken;
    behind[k] = s.given;
    length[k] = (unsigned)q[k].length;
    if (writes && r0 + k < a.requests) {
      const unsigned stored = stored_tokens(a, q[k], ring.got(s.taken, q[k].sums().taken));
      a.lengths_after[r0 + k] = (int)min(stored, 0x7fffffffu);
      a.row_start[r0 + k] = (int)token_of(s.tokens);
      unplaced += q[k].want - stored;
    }
    s = s + q[k].sums();
  }
  *reinterpret_cast<Four *>(to.row + r0) = row;
  *reinterpret_cast<Four *>(to.first + r0) = first;
  *reinterpret_cast<Four *>(to.behind + r0) = behind;
  *reinterpret_cast<Four *>(to.length + r0) = length;
  return before + total;
}

__device__ __forceinline__ void write_ends(const PageMapArgs &a, const Ring &ring, Sums all, long long unplaced) {
  a.row_start[a.requests] = (int)token_of(all.tokens);
  a.cursor_after[0] = a.cursor[0] + min(all.taken, ring.available);
  a.cursor_after[1] = a.cursor[1] + all.given;
  a.unplaced[0] = unplaced;
}

// the last of `starts`, ascending and from 0, that is not above `at`
__device__ __forceinline__ unsigned last_not_above(const unsigned *starts, unsigned n, unsigned at) {
  unsigned low = 0;
  for (unsigned step = 1u << (31 - __clz((int)n)); step; step >>= 1)
    if (low + step < n && starts[low + step] <= at) low += step;
  return low;
}

// The share of workgroup `group` of `groups` in the tokens, and in the pages given back.
template <int Threads>
__device__ __forceinline__ void fill(const PageMapArgs &a, const Ring &ring, Sums all, const Starts &of, unsigned group, unsigned groups) {
  const unsigned live = token_of(all.tokens), stride = groups * Threads;
  for (unsigned n = group * Threads + threadIdx.x; n < (a.tokens + kPerThread - 1) / kPerThread; n += stride) {
    const unsigned t0 = n * kPerThread;
    Vec<int, kPerThread> positions, requests;
    Vec<long long, kPerThread> slots;
    unsigned r = 0, start = 0, next = 0, k = ~0u;            // the request of the token, where it and the next one start, and its page
    unsigned length = 0, have = 0, first = 0, got = 0;
    int page = -1;
    if (t0 < live) r = last_not_above(of.row, a.requests, t0);
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const unsigned t = t0 + i;
      positions[i] = 0;
      requests[i] = -1;
      slots[i] = -1;
      if (t >= live) continue;
      if (t >= next) {                                       // the first token, or one of a request behind
        if (i > 0)
          do ++r;
          while (r + 1 < a.requests && of.row[r + 1] <= t);
        const bool more = r + 1 < a.requests;
        start = of.row[r];
        next = more ? of.row[r + 1] : live;
        length = of.length[r];
        first = of.first[r];
        got = ring.got(first, (more ? of.first[r + 1] : all.taken) - first);
        have = pages_of(a, length);
        k = ~0u;
      }
      const unsigned at = length + (t - start), on = at / a.page, offset = at - on * a.page;
      if (on != k) {
        k = on;
        page = -1;
        if (k < have) page = a.table[(long long)r * a.table_stride + k];
        else if (k < have + got) {
          page = a.pool[Ring::place(a, ring.head, first + (k - have))];
          if (offset == 0) a.table[(long long)r * a.table_stride + k] = page;        // the first token on a page enters it
        }
      }
      requests[i] = (int)r;
      positions[i] = (int)min(at, 0x7fffffffu);
      if (page >= 0) slots[i] = (long long)page * a.page + offset;
    }
    if (a.wide && t0 + kPerThread <= a.tokens) {
      *reinterpret_cast<Vec<int, kPerThread> *>(a.positions + t0) = positions;
      *reinterpret_cast<Vec<int, kPerThread> *>(a.request + t0) = requests;
      *reinterpret_cast<Vec<long long, 2> *>(a.slots + t0) = slots.xy;
      *reinterpret_cast<Vec<long long, 2> *>(a.slots + t0 + 2) = slots.zw;
      continue;
    }
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
      if (t0 + i < a.tokens) {
        a.positions[t0 + i] = positions[i];
        a.request[t0 + i] = requests[i];
        a.slots[t0 + i] = slots[i];
      }
  }
  if (a.entries == 0) return;
  // the pages of tokens that have no entry, which nobody above has seen: all pages taken, some a second time
  if (all.tokens > a.tokens)
    for (unsigned i = group * Threads + threadIdx.x; i < min(all.taken, ring.available); i += stride) {
      const unsigned r = last_not_above(of.first, a.requests, i);
      a.table[(long long)r * a.table_stride + pages_of(a, of.length[r]) + (i - of.first[r])] = a.pool[Ring::place(a, ring.head, i)];
    }
  for (unsigned i = group * Threads + threadIdx.x; i < min(all.given, a.entries); i += stride) {
    const unsigned r = last_not_above(of.behind, a.requests, i);
    const unsigned begin = of.behind[r], given = (r + 1 < a.requests ? of.behind[r + 1] : all.given) - begin, goal = pages_of(a, of.length[r]) - given;
    a.pool[Ring::place(a, ring.tail, i)] = a.table[(long long)r * a.table_stride + goal + (i - begin)];
  }
}

// The first workgroup writes what there is of each request, the others what there is of each token.
template <int Threads> __global__ __launch_bounds__(Threads) void page_map_kernel(PageMapArgs a) {
  constexpr int kRequests = Threads * kPerThread;
  __shared__ Four row[Threads], first[Threads], behind[Threads], length[Threads];
  static_assert(sizeof row == kRequests * sizeof(unsigned), "an entry a request");
  __shared__ Sums lds[Threads / kWave];
  __shared__ long long lds_sum[Threads / kWave];
  const Ring ring(a);
  const bool writes = blockIdx.x == 0;
  const Starts starts = {reinterpret_cast<unsigned *>(row), reinterpret_cast<unsigned *>(first), reinterpret_cast<unsigned *>(behind), reinterpret_cast<unsigned *>(length)};
  long long unplaced;
  const Sums all = scan_chunk<Threads>(a, ring, 0, Sums{0, 0, 0}, starts, writes, lds, unplaced);
  if (writes) {
    unplaced = block_sum<Threads>(unplaced, lds_sum);
    if (threadIdx.x == 0) write_ends(a, ring, all, unplaced);
    return;
  }
  __syncthreads();
  fill<Threads>(a, ring, all, starts, blockIdx.x - 1, gridDim.x - 1);
}

// sums of each chunk of requests, for the scan of the next kernel
__global__ __launch_bounds__(kMany) void page_map_sums_kernel(PageMapArgs a, Sums *sums) {
  __shared__ Sums lds[kMany / kWave];
  Sums mine = {0, 0, 0}, total;
  for (int k = 0; k < kPerThread; ++k) {
    const unsigned r = blockIdx.x * kChunk + k * kMany + threadIdx.x;
    if (r < a.requests) mine = mine + request_at(a, r).sums();
  }
  block_scan_exclusive<kMany>(mine, lds, total);
  if (threadIdx.x == 0) sums[blockIdx.x] = total;
}

__device__ __forceinline__ Sums sum_of_chunks(const Sums *sums, unsigned n, Sums *lds) {
  Sums mine = {0, 0, 0}, total;
  for (unsigned k = threadIdx.x; k < n; k += kMany) mine = mine + sums[k];
  block_scan_exclusive<kMany>(mine, lds, total);
  return total;
}

__global__ __launch_bounds__(kMany) void page_map_scan_kernel(PageMapArgs a, const Sums *sums, long long *unplaced_of, Starts starts) {
  __shared__ Sums lds[kMany / kWave];
  __shared__ long long lds_sum[kMany / kWave];
  const Ring ring(a);
  long long unplaced;
  scan_chunk<kMany>(a, ring, blockIdx.x * kChunk, sum_of_chunks(sums, blockIdx.x, lds), starts, true, lds, unplaced);
  unplaced = block_sum<kMany>(unplaced, lds_sum);
  if (threadIdx.x == 0) unplaced_of[blockIdx.x] = unplaced;
}

__global__ __launch_bounds__(kMany) void page_map_fill_kernel(PageMapArgs a, unsigned chunks, const Sums *sums, const long long *unplaced_of, Starts starts) {
  __shared__ Sums lds[kMany / kWave];
  __shared__ long long lds_sum[kMany / kWave];
  const Ring ring(a);
  const Sums all = sum_of_chunks(sums, chunks, lds);
  if (blockIdx.x == 0) {
    long long unplaced = 0;
    for (unsigned k = threadIdx.x; k < chunks; k += kMany) unplaced += unplaced_of[k];
    unplaced = block_sum<kMany>(unplaced, lds_sum);
    if (threadIdx.x == 0) write_ends(a, ring, all, unplaced);
  }
  fill<kMany>(a, ring, all, starts, blockIdx.x, gridDim.x);
}

struct PageMap final : Operator {
  PageMapArgs a;
  unsigned chunks() const { return ceil_div(a.requests, kChunk); }
  // what there is of each request (Starts), then each chunk's unplaced tokens and sums
  size_t workspace() const override {
    return a.requests <= (unsigned)kChunk ? 0 : chunks() * (4 * sizeof(unsigned) * kChunk + sizeof(long long) + sizeof(Sums));
  }
  void record(Recorder &r) const override {
    // as many workgroups as the tokens ask for, or the pages given back, which only the device knows, may ask for; one for each compute unit at
    // most: each sums all requests first
    auto groups = [&](int threads) { return std::min(std::max({ceil_div(a.tokens, threads * kPerThread), ceil_div(a.requests, kRequestsOfGroup), 1u}), 256u); };
    if (a.requests <= (unsigned)(kFew * kPerThread) && a.tokens <= 256u * kFew * kPerThread) {
      r.launch(&page_map_kernel<kFew>, groups(kFew) + 1, kFew, a);
      return;
    }
    if (a.requests <= (unsigned)kChunk) {
      r.launch(&page_map_kernel<kMany>, groups(kMany) + 1, kMany, a);
      return;
    }
    const size_t entries = (size_t)chunks() * kChunk;
    unsigned *row = reinterpret_cast<unsigned *>(r.workspace);
    const Starts starts = {row, row + entries, row + 2 * entries, row + 3 * entries};
    long long *unplaced_of = reinterpret_cast<long long *>(row + 4 * entries);
    Sums *sums = reinterpret_cast<Sums *>(unplaced_of + chunks());
    r.launch(&page_map_sums_kernel, chunks(), kMany, a, sums);
    r.launch(&page_map_scan_kernel, chunks(), kMany, a, sums, unplaced_of, starts);
    r.launch(&page_map_fill_kernel, groups(kMany), kMany, a, chunks(), sums, unplaced_of, starts);
  }
  const char *name() const override { return "page map"; }
};

}  // namespace

int make_page_map(const fc_page_map &a, std::unique_ptr<Operator> &out, std::string &err) {
  TensorChecks c(err);
  c.array("lengths", a.lengths, FC_I32, {-1});
  const int64_t requests = a.lengths.shape[0];
  c.array("new_tokens", a.new_tokens, FC_I32, {requests});
  c.array("pool", a.pool, FC_I32, {-1}, true);
  c.array("cursor", a.cursor, FC_I64, {2});
  c.array("table", a.table, FC_I32, {requests, -1}, true);
  c.array("lengths_after", a.lengths_after, FC_I32, {requests}, true);
  c.array("row_start", a.row_start, FC_I32, {requests + 1}, true);
  c.array("slots", a.slots, FC_I64, {-1}, true);
  c.array("positions", a.positions, FC_I32, {a.slots.shape[0]}, true);
  c.array("request", a.request, FC_I32, {a.slots.shape[0]}, true);
  c.array("cursor_after", a.cursor_after, FC_I64, {2}, true);
  c.array("unplaced", a.unplaced, FC_I64, {1}, true);
  if (!c.ok()) return c.code();
  if (a.page_size < 1) return c.fail(FC_E_ARG, "page_size must be positive").code();
  if (requests * a.table.shape[1] > 0x7fffffff) return c.fail(FC_E_LIMIT, "table has more than 2^31-1 entries").code();
  auto op = std::make_unique<PageMap>();
  PageMapArgs &k = op->a;
  k.lengths = static_cast<const int *>(a.lengths.ptr);
  k.fresh = static_cast<const int *>(a.new_tokens.ptr);
  k.pool = static_cast<int *>(a.pool.ptr);
  k.cursor = static_cast<const long long *>(a.cursor.ptr);
  k.table = static_cast<int *>(a.table.ptr);
  k.lengths_after = static_cast<int *>(a.lengths_after.ptr);
  k.row_start = static_cast<int *>(a.row_start.ptr);
  k.slots = static_cast<long long *>(a.slots.ptr);
  k.positions = static_cast<int *>(a.positions.ptr);
  k.request = static_cast<int *>(a.request.ptr);
  k.cursor_after = static_cast<long long *>(a.cursor_after.ptr);
  k.unplaced = static_cast<long long *>(a.unplaced.ptr);
  k.table_stride = a.table.stride[0];
  k.wide = common_alignment(a.lengths, 4) == 4 && common_alignment(a.new_tokens, 4) == 4 && common_alignment(a.slots, 2) == 2 &&
           common_alignment(a.positions, 4) == 4 && common_alignment(a.request, 4) == 4;
  k.requests = (unsigned)requests;
  k.width = (unsigned)a.table.shape[1];
  k.page = (unsigned)a.page_size;
  k.tokens = (unsigned)a.slots.shape[0];
  k.entries = (unsigned)a.pool.shape[0];
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
