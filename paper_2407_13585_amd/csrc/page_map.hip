// Block tables and slot maps of one step of a server (include/fc.h, fc_page_map).
//
// Three prefix sums over the requests (new tokens, pages taken, pages given back), then every token finds its request by
// bisection in the first of them, and with it its position and page: a scan, two gathers and two scatters, and nothing between
// them but the sums.  The bytes are few (16 a token, 20 a request), so a step costs its launches and the chain of dependent reads
// of one token.  Up to kInLds requests every workgroup sums all of them for itself and keeps the sums in LDS, which makes a
// step one launch; above, two kernels leave the sums in scratch for the third.
#include "operators.hpp"

namespace fc {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kPerThread = 4;
constexpr int kChunk = kThreads * kPerThread;      // requests that a workgroup sums at once
constexpr int kInLds = kChunk;

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
};

struct Sums {
  long long tokens;
  int taken, given;                                // at most the entries of the table, which are below 2^31
};
__device__ __forceinline__ Sums operator+(Sums a, Sums b) { return {a.tokens + b.tokens, a.taken + b.taken, a.given + b.given}; }

struct Request {
  int length, fresh;
  unsigned want, have, goal;                       // want: below 2^32, the sum of two values below 2^31
  __device__ __forceinline__ Sums sums() const { return {fresh > 0 ? fresh : 0, goal > have ? (int)(goal - have) : 0, have > goal ? (int)(have - goal) : 0}; }
};

__device__ __forceinline__ unsigned pages_of(const PageMapArgs &a, unsigned n) {
  const unsigned q = n / a.page;
  return min(q + (n != q * a.page ? 1u : 0u), a.width);
}

__device__ __forceinline__ Request request_at(const PageMapArgs &a, unsigned r) {
  Request q;
  q.length = max(a.lengths[r], 0);
  q.fresh = a.fresh[r];
  const long long want = (long long)q.length + q.fresh;
  q.want = want > 0 ? (unsigned)want : 0u;
  q.have = pages_of(a, (unsigned)q.length);
  q.goal = pages_of(a, q.want);
  return q;
}

// The ring of free pages, at places counted from the cursor's own.
struct Ring {
  unsigned head, tail, available;
  __device__ __forceinline__ Ring(const PageMapArgs &a) {
    const long long h = a.cursor[0], t = a.cursor[1], n = a.entries;
    available = (unsigned)min(max(t - h, 0ll), n);
    head = n ? (unsigned)((h % n + n) % n) : 0u;
    tail = n ? (unsigned)((t % n + n) % n) : 0u;
  }
  // `k` below the number of entries
  static __device__ __forceinline__ unsigned place(const PageMapArgs &a, unsigned from, unsigned k) {
    const unsigned p = from + k;                   // both below 2^31
    return p >= a.entries ? p - a.entries : p;
  }
  __device__ __forceinline__ unsigned got(int first, int taken) const {
    return (unsigned)first < available ? min(available - (unsigned)first, (unsigned)taken) : 0u;
  }
};

__device__ __forceinline__ unsigned stored_tokens(const PageMapArgs &a, const Request &q, unsigned got) {
  const unsigned long long room = (unsigned long long)(q.fresh > 0 ? q.have + got : a.width) * a.page;
  return (unsigned)min((unsigned long long)q.want, room);
}

__device__ __forceinline__ Sums wave_scan(Sums v) {
  v.taken = wave_scan_inclusive<AddI32>(v.taken);
  v.given = wave_scan_inclusive<AddI32>(v.given);
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const long long u = __shfl_up(v.tokens, d);
    if (lane_id() >= d) v.tokens += u;
  }
  return v;
}

// Sums of the threads before this one; total: of all.  lds: kWaves entries, free when the call returns.
__device__ __forceinline__ Sums block_scan_exclusive(Sums v, Sums *lds, Sums &total) {
  const Sums upto = wave_scan(v);
  __syncthreads();
  if (lane_id() == kWave - 1) lds[wave_id()] = upto;
  __syncthreads();
  Sums before = {0, 0, 0};
  total = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave_id()) before = before + lds[w];
    total = total + lds[w];
  }
  __syncthreads();
  return {before.tokens + upto.tokens - v.tokens, before.taken + upto.taken - v.taken, before.given + upto.given - v.given};
}

__device__ __forceinline__ long long block_sum(long long v, long long *lds) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
  __syncthreads();
  if (lane_id() == 0) lds[wave_id()] = v;
  __syncthreads();
  long long sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += lds[w];
  return sum;
}

__device__ __forceinline__ int saturated(long long tokens) { return tokens > 0x7fffffff ? 0x7fffffff : (int)tokens; }

// The sums before each request of [begin, begin + kChunk), the first at row[begin] and so on, what comes before them added; the
// arrays of one entry a request are written too where `writes`.  Returns the sums up to the end, and the chunk's unplaced tokens.
__device__ __forceinline__ Sums scan_chunk(const PageMapArgs &a, const Ring &ring, unsigned begin, Sums before, int *row, int *first, int *behind,
                                           bool writes, Sums *lds, long long &unplaced) {
  Request q[kPerThread];
  Sums mine = {0, 0, 0};
  const unsigned r0 = begin + threadIdx.x * kPerThread;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k)
    if (r0 + k < a.requests) {
      q[k] = request_at(a, r0 + k);
      mine = mine + q[k].sums();
    }
  Sums total;
  Sums s = before + block_scan_exclusive(mine, lds, total);
  unplaced = 0;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k)
    if (r0 + k < a.requests) {
      row[r0 + k] = saturated(s.tokens);
      first[r0 + k] = s.taken;
      behind[r0 + k] = s.given;
      if (writes) {
        const unsigned stored = stored_tokens(a, q[k], ring.got(s.taken, q[k].sums().taken));
        a.lengths_after[r0 + k] = (int)min(stored, 0x7fffffffu);
        a.row_start[r0 + k] = saturated(s.tokens);
        unplaced += q[k].want - stored;
      }
      s = s + q[k].sums();
    }
  return before + total;
}

__device__ __forceinline__ void write_ends(const PageMapArgs &a, const Ring &ring, Sums all, long long unplaced) {
  a.row_start[a.requests] = saturated(all.tokens);
  a.cursor_after[0] = a.cursor[0] + min((unsigned)all.taken, ring.available);
  a.cursor_after[1] = a.cursor[1] + all.given;
  a.unplaced[0] = unplaced;
}

// the last of `starts`, ascending and from 0, that is not above `at`
__device__ __forceinline__ unsigned last_not_above(const int *starts, unsigned n, int at) {
  unsigned low = 0;
  for (unsigned step = 1u << (31 - __clz((int)n)); step; step >>= 1)
    if (low + step < n && starts[low + step] <= at) low += step;
  return low;
}

// This workgroup's share of the tokens, and of the pages given back.
__device__ __forceinline__ void fill(const PageMapArgs &a, const Ring &ring, Sums all, const int *row, const int *first, const int *behind) {
  const unsigned stride = gridDim.x * kThreads;
  // also tokens that have no entry: the first on a page still enters it
  const unsigned live = (unsigned)saturated(all.tokens);
  for (unsigned t = blockIdx.x * kThreads + threadIdx.x; t < max(a.tokens, live); t += stride) {
    int position = 0, request = -1;
    long long slot = -1;
    if (t < live) {
      const unsigned r = last_not_above(row, a.requests, (int)t);
      const Request q = request_at(a, r);
      const unsigned at = (unsigned)q.length + (t - (unsigned)row[r]);
      const unsigned k = at / a.page, offset = at - k * a.page, got = ring.got(first[r], q.sums().taken);
      request = (int)r;
      position = (int)min(at, 0x7fffffffu);
      int page = -1;
      if (k < q.have) page = a.table[(long long)r * a.table_stride + k];
      else if (k < q.have + got) {
        page = a.pool[Ring::place(a, ring.head, (unsigned)first[r] + (k - q.have))];
        if (offset == 0) a.table[(long long)r * a.table_stride + k] = page;      // the first token on a page enters it
      }
      if (page >= 0) slot = (long long)page * a.page + offset;
    }
    if (t >= a.tokens) continue;
    a.positions[t] = position;
    a.request[t] = request;
    a.slots[t] = slot;
  }
  if (a.entries == 0) return;
  for (unsigned i = blockIdx.x * kThreads + threadIdx.x; i < min((unsigned)all.given, a.entries); i += stride) {
    const unsigned r = last_not_above(behind, a.requests, (int)i);
    const Request q = request_at(a, r);
    a.pool[Ring::place(a, ring.tail, i)] = a.table[(long long)r * a.table_stride + q.goal + (i - (unsigned)behind[r])];
  }
}

__global__ __launch_bounds__(kThreads) void page_map_kernel(PageMapArgs a) {
  __shared__ int row[kInLds], first[kInLds], behind[kInLds];
  __shared__ Sums lds[kWaves];
  __shared__ long long lds_sum[kWaves];
  const Ring ring(a);
  const bool writes = blockIdx.x == 0;
  long long unplaced;
  const Sums all = scan_chunk(a, ring, 0, Sums{0, 0, 0}, row, first, behind, writes, lds, unplaced);
  if (writes) {
    unplaced = block_sum(unplaced, lds_sum);
    if (threadIdx.x == 0) write_ends(a, ring, all, unplaced);
  }
  __syncthreads();
  fill(a, ring, all, row, first, behind);
}

// sums of each chunk of requests, for the scan of the next kernel
__global__ __launch_bounds__(kThreads) void page_map_sums_kernel(PageMapArgs a, Sums *sums) {
  __shared__ Sums lds[kWaves];
  Sums mine = {0, 0, 0}, total;
  for (int k = 0; k < kPerThread; ++k) {
    const unsigned r = blockIdx.x * kChunk + k * kThreads + threadIdx.x;
    if (r < a.requests) mine = mine + request_at(a, r).sums();
  }
  block_scan_exclusive(mine, lds, total);
  if (threadIdx.x == 0) sums[blockIdx.x] = total;
}

__device__ __forceinline__ Sums sum_of_chunks(const Sums *sums, unsigned n, Sums *lds) {
  Sums mine = {0, 0, 0}, total;
  for (unsigned k = threadIdx.x; k < n; k += kThreads) mine = mine + sums[k];
  block_scan_exclusive(mine, lds, total);
  return total;
}

__global__ __launch_bounds__(kThreads) void page_map_scan_kernel(PageMapArgs a, const Sums *sums, long long *unplaced_of, int *row, int *first, int *behind) {
  __shared__ Sums lds[kWaves];
  __shared__ long long lds_sum[kWaves];
  const Ring ring(a);
  long long unplaced;
  scan_chunk(a, ring, blockIdx.x * kChunk, sum_of_chunks(sums, blockIdx.x, lds), row, first, behind, true, lds, unplaced);
  unplaced = block_sum(unplaced, lds_sum);
  if (threadIdx.x == 0) unplaced_of[blockIdx.x] = unplaced;
}

__global__ __launch_bounds__(kThreads) void page_map_fill_kernel(PageMapArgs a, unsigned chunks, const Sums *sums, const long long *unplaced_of, const int *row,
                                                                 const int *first, const int *behind) {
  __shared__ Sums lds[kWaves];
  __shared__ long long lds_sum[kWaves];
  const Ring ring(a);
  const Sums all = sum_of_chunks(sums, chunks, lds);
  if (blockIdx.x == 0) {
    long long unplaced = 0;
    for (unsigned k = threadIdx.x; k < chunks; k += kThreads) unplaced += unplaced_of[k];
    unplaced = block_sum(unplaced, lds_sum);
    if (threadIdx.x == 0) write_ends(a, ring, all, unplaced);
  }
  fill(a, ring, all, row, first, behind);
}

struct PageMap final : Operator {
  PageMapArgs a;
  unsigned chunks() const { return ceil_div(a.requests, kChunk); }
  // each chunk's sums and unplaced tokens, then the sums before each request
  size_t workspace() const override {
    return a.requests <= (unsigned)kInLds ? 0 : chunks() * (sizeof(Sums) + sizeof(long long)) + 3 * sizeof(int) * (size_t)a.requests;
  }
  void record(Recorder &r) const override {
    // tokens, and what is given back, which only the device knows: as many workgroups as the tokens ask for, one for each
    // compute unit at most (each sums all requests first)
    const unsigned grid = std::min(std::max(ceil_div(a.tokens, kThreads), 1u), 256u);
    if (a.requests <= (unsigned)kInLds) {
      r.launch(&page_map_kernel, grid, kThreads, a);
      return;
    }
    Sums *sums = reinterpret_cast<Sums *>(r.workspace);
    long long *unplaced_of = reinterpret_cast<long long *>(sums + chunks());
    int *row = reinterpret_cast<int *>(unplaced_of + chunks()), *first = row + a.requests, *behind = first + a.requests;
    r.launch(&page_map_sums_kernel, chunks(), kThreads, a, sums);
    r.launch(&page_map_scan_kernel, chunks(), kThreads, a, sums, unplaced_of, row, first, behind);
    r.launch(&page_map_fill_kernel, grid, kThreads, a, chunks(), sums, unplaced_of, row, first, behind);
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
  k.requests = (unsigned)requests;
  k.width = (unsigned)a.table.shape[1];
  k.page = (unsigned)a.page_size;
  k.tokens = (unsigned)a.slots.shape[0];
  k.entries = (unsigned)a.pool.shape[0];
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
