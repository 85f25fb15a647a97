// The pages of a request that count most for a key head (include/fc.h, fc_page_select).
//
// No key of a page scores more with q than  s = sum over d of max(q_d, 0) high_d + min(q_d, 0) low_d,  which is a matrix product: bounds of
// pages are its rows, the query heads of a group its columns.  Its sums are of 64 bits, as is the matrix instruction: which of two pages is taken must not
// depend on the order in which they were added up.  Of the s of a group's heads the largest counts.
//
// The scores become whole numbers of 64 bits in the same order; the k-th largest is found from its upper digits down, 8 bits at a time, from
// the first that differs between the least and the largest on, until the pages above and at it are as many as are wanted.  One workgroup does it
// for a request and key head (a row); where rows are few and their pages many, a row's scores are split into pieces of about the same size, and the last
// workgroup to be done selects.
//
// What bounds it.  One request of 4096 pages of 8 key heads of 128, 64 heads (bf16, 17 MB) 28 us: 5 to the row's workgroup and its table, 8 for the scores
// (reads 4, arithmetic 4, each once and one behind the other), 3 to hand them to one workgroup, the rest that workgroup alone, step after step.  64 requests of up to 1024 pages, 8
// key heads of 128, 32 heads (bf16, 134 MB) 56 us: without selection 48.5, without most of the arithmetic too 42.5, without the table's reads 35, so
// 3.8 TB/s of what it must read; 300 requests of 900 pages (bf16, 1.1 GB) 250 us, 4.4 TB/s, in 32 bits 442 us, 5.0 TB/s.  4 short requests 3.8 us: the launch.
#include "operators.hpp"

#include <algorithm>

namespace fc {

namespace {

// Threads of a workgroup.  Many: where long rows are split, of which one workgroup orders all scores.  us by many and by few, 8 key heads of 128, groups of 8 (bf16): one
// request of 2100 pages 28.5 and 27.6, of 3000 28.9 and 31.1, of 6000 31 and 39, of 16000 66 and 118; 32 requests of 2100 pages 106 and 119, of 6000 276 and
// 300.  Short rows leave their waves idle: 8 requests of 500 pages 26 and 16, 64 of 1024 78 and 68.  The width of the table decides, since lengths lie on the device: a table
// that is much wider than its requests are long costs what this says.  Widths of 2048 entries at most and of more: 8 requests of 500 pages, groups of 8, 17 and 24.5
// us, 64 of 1 to 1024 pages, groups of 4, 56 and 78, 64 of 16 pages 3.6 (17 entries) and 15 (4097).
constexpr int kFew = 256, kMany = 1024;
// of 16 pages, that a wave reads before it scores them: two take 67 us where one takes 61 (64 ragged requests), 15.4 and 12.5 (19 in f32)
constexpr int kTilesOfWave = 1;
constexpr unsigned block_pages(int threads) { return 16 * kTilesOfWave * threads / kWave; }       // of a row that a workgroup scores at a time
constexpr unsigned kKept = 1024;                             // keys that stay in LDS where one workgroup has a whole row (300 requests of 900 pages 245 us, 264 by memory)
constexpr unsigned kListed = 2048;                           // selected positions that are put in order in LDS
constexpr unsigned long long kAlways = ~0ull;                // above every score; 0, below every score, is a page that is not there

struct SelectArgs {
  const char *q, *bounds;
  const int *table, *lengths;
  int *selected, *selected_lengths;
  unsigned long long *keys;                // DEVICE: of each row `width`; NULL: they fit LDS
  unsigned *counters;                      // DEVICE: one a row, 0 between launches
  long long q_request, q_head, b_page, b_head, b_half, table_stride, s_request, s_head, l_request;
  unsigned requests, heads, group, dim, page, pages, width, most, first, last;
  unsigned pieces;                         // of about the same size that all rows together are split into, and one more a row; 0: they are not
};

// a number that orders scores as they are; NaN counts as infinite, -0 as 0
__device__ __forceinline__ unsigned long long key_of(double s) {
  s = s != s ? __builtin_inf() : s + 0.0;
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, s);
  return bits >> 63 ? ~bits : bits | 1ull << 63;
}

// the value of another lane of the four
template <int Ctrl> __device__ __forceinline__ double of_four(double v) {
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, v);
  const unsigned low = (unsigned)dpp_move<Ctrl>(0, (int)(unsigned)bits), high = (unsigned)dpp_move<Ctrl>(0, (int)(unsigned)(bits >> 32));
  return __builtin_bit_cast(double, (unsigned long long)high << 32 | low);
}

// Scores of pages for the query heads of a key head.  The instruction has four products of 4 pages, 4 elements and 4 heads: lane (r, g), r = lane % 16,
// g = lane / 16, holds elements of page r, and of query head r % 4 the same ones; lane (4 n + j, i) gets page 4 n + i and head j.
// HeadTiles: four query heads each that are taken together; groups of more than four take two at a time (32 requests of 2000 pages, groups of 8: 106 us, 126
// with one), others one, whose second would be empty (64 of 1024 pages, groups of 4: 70 us, 98 with two).
// Whole: the elements of a head fill the lanes' reads (32 requests of 2000 pages 106 us, 142 with the tests that other heads need).
template <class T, int HeadTiles, bool Whole> struct Scores {
  static constexpr int N = 16 / sizeof(T), kChunks = 4, kTiles = kTilesOfWave;  // 16 bytes of each of four lanes; of them, and of 16 pages, under way
  using Part = Vec<T, N>;
  const SelectArgs &a;
  const T *q, *bounds;
  const int *table;
  unsigned r, g;

  __device__ __forceinline__ Scores(const SelectArgs &args, const T *queries, const T *of_head, const int *pages)
      : a(args), q(queries), bounds(of_head), table(pages), r(lane_id() & 15), g(lane_id() >> 4) {}

  // all reads are made, so that none waits for a condition: past the end of a head they are of its last elements, and then cleared
  static __device__ __forceinline__ Part load(const T *from, unsigned d, unsigned dim) { return load_vec<T, N>(from + (Whole ? d : min(d, dim - N))); }
  static __device__ __forceinline__ void clear(Part &x, bool inside) {
    if constexpr (!Whole)
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = inside ? x[e] : (T)0.0f;
  }

  // use(position, is it there, score, is it the first) for the 16 kTiles pages from `at` on that lie below `end`, for every 4 HeadTiles query heads
  template <class Use> __device__ __forceinline__ void run(unsigned at, unsigned end, Use &&use) {
    if (at >= end) return;
    const T *row[kTiles];
    unsigned long long there[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const unsigned w = at + 16 * t + r, page = (unsigned)table[min(w, end - 1)];
      const bool is_there = w < end && page < a.pages;
      there[t] = __ballot(is_there);
      row[t] = bounds + (is_there ? page * a.b_page : 0ll);
    }
    for (unsigned head0 = 0; head0 < a.group; head0 += 4 * HeadTiles) {
      const T *from[HeadTiles];
      bool mine[HeadTiles], nan[HeadTiles];
      double up[kTiles][HeadTiles], down[kTiles][HeadTiles];
#pragma unroll
      for (int n = 0; n < HeadTiles; ++n) {
        const unsigned head = head0 + 4 * n + (r & 3);
        mine[n] = head < a.group;
        from[n] = q + (mine[n] ? head * a.q_head : 0ll);
        nan[n] = false;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) up[t][n] = down[t][n] = 0.0;
      }
      for (unsigned d0 = g * N; d0 < a.dim + g * N; d0 += 4 * N * kChunks) {
        Part x[HeadTiles][kChunks], l[kTiles][kChunks], h[kTiles][kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          const unsigned d = d0 + 4 * N * c;
          if (d - g * N >= a.dim) break;                     // the same for all lanes
#pragma unroll
          for (int n = 0; n < HeadTiles; ++n) x[n][c] = load(from[n], d, a.dim);
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            h[t][c] = load(row[t] + a.b_half, d, a.dim);
            l[t][c] = load(row[t], d, a.dim);
          }
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          const unsigned d = d0 + 4 * N * c;
          if (d - g * N >= a.dim) break;
#pragma unroll
          for (int n = 0; n < HeadTiles; ++n) clear(x[n][c], d < a.dim);
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            clear(h[t][c], d < a.dim);
            clear(l[t][c], d < a.dim);
          }
#pragma unroll
          for (int e = 0; e < N; ++e) {
            double high[kTiles], low[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
              high[t] = (double)(float)h[t][c][e];
              low[t] = (double)(float)l[t][c][e];
            }
#pragma unroll
            for (int n = 0; n < HeadTiles; ++n) {
              const float v = (float)x[n][c][e];
              nan[n] |= v != v;                              // which the maxima and minima would lose
              const double plus = (double)fmaxf(v, 0.0f), minus = (double)fminf(v, 0.0f);
#pragma unroll
              for (int t = 0; t < kTiles; ++t) {
                up[t][n] = __builtin_amdgcn_mfma_f64_4x4x4f64(high[t], plus, up[t][n], 0, 0, 0);
                down[t][n] = __builtin_amdgcn_mfma_f64_4x4x4f64(low[t], minus, down[t][n], 0, 0, 0);
              }
            }
          }
        }
      }
#pragma unroll
      for (int n = 0; n < HeadTiles; ++n) nan[n] = (__ballot(nan[n]) & (0x1111111111111111ull << (r & 3))) != 0;       // of all lanes of the head
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        double best = -__builtin_inf();
#pragma unroll
        for (int n = 0; n < HeadTiles; ++n) {
          const double s = up[t][n] + down[t][n];
          if (mine[n]) best = fmax(best, s != s || nan[n] ? __builtin_inf() : s);
        }
        best = fmax(best, of_four<0xb1>(best));              // quad_perm 1,0,3,2
        best = fmax(best, of_four<0x4e>(best));              // quad_perm 2,3,0,1
        const unsigned i = (r >> 2) * 4 + g, w = at + 16 * t + i;
        if ((r & 3) == 0 && w < end) use(w, (there[t] >> i & 1) != 0, best, head0 == 0);
      }
    }
  }
};

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

// The sums of two numbers that a wave's lanes share, over the waves before this one and in all.
struct Sums {
  unsigned x, y, all_x, all_y;
};
template <int Waves> __device__ __forceinline__ Sums sum_of_waves(unsigned x, unsigned y, unsigned (*lds)[2]) {
  if (lane_id() == 0) { lds[wave_id()][0] = x; lds[wave_id()][1] = y; }
  __syncthreads();
  Sums s{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < Waves; ++w) {
    if (w < wave_id()) { s.x += lds[w][0]; s.y += lds[w][1]; }
    s.all_x += lds[w][0];
    s.all_y += lds[w][1];
  }
  return s;
}
__device__ __forceinline__ unsigned lanes_of(bool b) { return (unsigned)__popcll(__ballot(b)); }
// the lanes of `mask` before this one
__device__ __forceinline__ unsigned lanes_before(unsigned long long mask) { return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u)); }

__device__ __forceinline__ unsigned length_of(const SelectArgs &a, int length) { return (unsigned)min((unsigned long long)max(length, 0), (unsigned long long)a.width * a.page); }
__device__ __forceinline__ unsigned pages_of(const SelectArgs &a, unsigned length) { return (length + a.page - 1) / a.page; }
// no more pages than are wanted: all that are there are taken
__device__ __forceinline__ bool is_scored(const SelectArgs &a, unsigned count) { return count > a.most && a.pages > 0; }
// of a row: as many pages as a workgroup scores at a time, or one
template <int Threads> __device__ __forceinline__ unsigned units_of(const SelectArgs &a, unsigned count) { return is_scored(a, count) ? (count - 1) / block_pages(Threads) + 1 : 1u; }

// Scores the units [unit0, unit1) of the row of request b and key head `head`; the last of the `parts` workgroups that it is split over, who count on
// `counter`, then selects.
// Held: keys of a row that a lane keeps in registers, no more than a call's tables need; 0: as many as there are, read again whenever they are looked at
// (32 requests of 2000 pages 106 us, 112 without, 118 with registers for four times as many).
template <class T, int HeadTiles, bool Whole, int Held, int Threads>
__device__ __forceinline__ void select_of_row(const SelectArgs &a, unsigned b, unsigned head, unsigned length, unsigned unit0, unsigned unit1, unsigned parts, unsigned *counter) {
  constexpr int kWaves = Threads / kWave;
  constexpr unsigned kBlock = block_pages(Threads);
  __shared__ unsigned long long kept[kKept];
  __shared__ unsigned counts[2][256], sums[2][kWaves][2], found[2][3];
  __shared__ int ends[2][kWaves];
  __shared__ unsigned listed[kListed];
  const unsigned count = pages_of(a, length);
  const int *const table = a.table + b * a.table_stride;
  int *const selected = a.selected + b * a.s_request + head * a.s_head;
  unsigned long long *const far = a.keys ? a.keys + (size_t)(b * a.heads + head) * a.width : nullptr;
  const bool scored = is_scored(a, count);
  const bool near = parts == 1 && count <= kKept;            // the keys never leave LDS
  // a wave has `each` times 64 positions side by side, a lane one of every 64
  const unsigned each = (count + Threads - 1) / Threads, w0 = (unsigned)wave_id() * each * kWave + lane_id();
  if (scored) {
    const T *const q = reinterpret_cast<const T *>(a.q) + b * a.q_request + head * a.group * a.q_head;
    const T *const bounds = reinterpret_cast<const T *>(a.bounds) + head * a.b_head;
    Scores<T, HeadTiles, Whole> scores(a, q, bounds, table);
    for (unsigned at = unit0 * kBlock; at < min(unit1 * kBlock, count); at += kBlock)
      scores.run(at + kBlock / kWaves * (unsigned)wave_id(), min(at + kBlock, count), [&](unsigned w, bool there, double s, bool first) {
        unsigned long long key = !there ? 0ull : w < a.first || w + a.last >= count ? kAlways : key_of(s);
        if (near) kept[w] = first ? key : max(kept[w], key);
        else {
          unsigned long long *const to = far + w;
          store_agent64(to, first ? key : max(load_agent64(to), key));
        }
      });
  }
  if (parts > 1) {
    if (!last_to_arrive(counter, parts)) return;
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  // N keys from the lane's i0-th on, all read before the first is waited for; 0 behind its last
  auto read_keys = [&](unsigned i0, auto &to) {
    constexpr int n = sizeof(to) / sizeof(to[0]);
    if (!scored) {
      unsigned page[n];
#pragma unroll
      for (int i = 0; i < n; ++i)
        if (i0 + i < each) page[i] = (unsigned)table[min(w0 + (i0 + i) * kWave, count - 1)];
#pragma unroll
      for (int i = 0; i < n; ++i) to[i] = i0 + i < each && w0 + (i0 + i) * kWave < count && page[i] < a.pages ? kAlways : 0ull;
    } else {
      if (near)
#pragma unroll
        for (int i = 0; i < n; ++i) to[i] = kept[min(w0 + (i0 + i) * kWave, count - 1)];
      else
#pragma unroll
        for (int i = 0; i < n; ++i)
          if (i0 + i < each) to[i] = load_agent64(far + min(w0 + (i0 + i) * kWave, count - 1));
#pragma unroll
      for (int i = 0; i < n; ++i) to[i] = i0 + i < each && w0 + (i0 + i) * kWave < count ? to[i] : 0ull;
    }
  };
  unsigned long long held[Held ? Held : 1];
  if constexpr (Held > 0) read_keys(0, held);
  // use(position, key) by all lanes together
  auto for_keys = [&](auto &&use) {
    if constexpr (Held > 0) {
#pragma unroll
      for (int i = 0; i < Held; ++i)
        if ((unsigned)i < each) use(w0 + i * kWave, held[i]);
    } else {
      for (unsigned i0 = 0; i0 < each; i0 += 8) {
        unsigned long long some[8];
        read_keys(i0, some);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i0 + i < each) use(w0 + (i0 + i) * kWave, some[i]);
      }
    }
  };

  // taken: keys above `bar` with their lowest `shift` bits cut off, and of those at it the first `level`
  unsigned long long bar = ~0ull;
  unsigned shift = 0, level = 0, turn = 0;
  bool all = true;
  if (scored) {
    // the upper halves of the keys, as signed numbers in the same order: the least, turned round, and the largest
    int least = INT32_MIN, largest = INT32_MIN;
    unsigned mine = 0, always = 0;
    for_keys([&](unsigned, unsigned long long key) {
      mine += lanes_of(key != 0);
      always += lanes_of(key == kAlways);
      if (key != 0 && key != kAlways) {
        const int upper = (int)((unsigned)(key >> 32) ^ 0x80000000u);
        least = max(least, ~upper);
        largest = max(largest, upper);
      }
    });
    least = wave_reduce<MaxI32>(least);
    largest = wave_reduce<MaxI32>(largest);
    if (lane_id() == 0) { ends[0][wave_id()] = least; ends[1][wave_id()] = largest; }
    if (threadIdx.x < 256) counts[0][threadIdx.x] = 0;
    const Sums there = sum_of_waves<kWaves>(mine, always, sums[turn]);
    turn ^= 1;
    all = there.all_x <= a.most;
    const unsigned wanted = a.most - min(there.all_y, a.most);                 // of those that are not taken anyway
    if (!all && wanted > 0) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) { least = max(least, ends[0][w]); largest = max(largest, ends[1][w]); }
      const unsigned upper = (unsigned)largest ^ 0x80000000u, differ = (unsigned)(~least ^ largest);
      shift = differ ? 64u - (unsigned)__clz((int)differ) : 32u;               // keys differ below
      bar = shift == 64 ? 0 : (unsigned long long)upper << 32 >> shift;
      level = wanted;
      for (unsigned n = 0; shift > 0; n ^= 1) {
        const unsigned digit = min(shift, 8u), upper = shift;
        shift -= digit;
        for_keys([&](unsigned, unsigned long long key) {
          if (key != 0 && key != kAlways && (upper == 64 ? 0 : key >> upper) == bar) atomicAdd(&counts[n][key >> shift & ((1u << digit) - 1)], 1u);
        });
        __syncthreads();
        if (wave_id() == 0) {                                                  // from the largest digit down: the one where `level` is reached
          unsigned here[4], mine4 = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) mine4 += here[i] = counts[n][255 - (4 * lane_id() + i)];
          unsigned upto = (unsigned)wave_scan_inclusive<AddI32>((int)mine4) - mine4;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (level > upto && level <= upto + here[i]) {
              found[n][0] = 255 - (4 * lane_id() + i);
              found[n][1] = upto;
              found[n][2] = here[i];
            }
            upto += here[i];
          }
        } else if (wave_id() == 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) counts[n ^ 1][4 * lane_id() + i] = 0;
        }
        __syncthreads();
        bar = bar << digit | found[n][0];
        level -= found[n][1];
        if (level == found[n][2]) break;                                       // all of them are taken
      }
    }
  }
  // the bar's keys are those from `low` up to `high`
  const unsigned long long low = bar << shift, high = low + ((1ull << shift) - 1);
  unsigned above = 0, at_bar = 0;
  for_keys([&](unsigned, unsigned long long key) {
    const bool over = key > high || (all && key != 0) || key == kAlways;
    above += lanes_of(over);
    at_bar += lanes_of(!over && key != 0 && key >= low);
  });
  const Sums to = sum_of_waves<kWaves>(above, at_bar, sums[turn]);
  unsigned at_before = to.y, slot0 = to.x + min(at_before, level);
  const unsigned taken = min(to.all_x + min(to.all_y, level), a.most);
  bool is_last = false;
  for_keys([&](unsigned w, unsigned long long key) {
    const bool over = key > high || (all && key != 0) || key == kAlways;
    const bool at = !over && key != 0 && key >= low;
    const unsigned long long equal = __ballot(at);
    const bool take = over || (at && at_before + lanes_before(equal) < level);
    const unsigned long long mask = __ballot(take);
    const unsigned slot = slot0 + lanes_before(mask);
    if (take && slot < a.most) {
      if (slot < kListed) listed[slot] = w;
      else selected[slot] = table[w];
      is_last |= w + 1 == count;
    }
    at_before += (unsigned)__popcll(equal);
    slot0 += (unsigned)__popcll(mask);
  });
  const unsigned short_of = __syncthreads_or(is_last) ? count * a.page - length : 0u;
  for (unsigned k = threadIdx.x; k < min(taken, kListed); k += Threads) selected[k] = table[listed[k]];
  for (unsigned k = taken + threadIdx.x; k < a.most; k += Threads) selected[k] = -1;
  if (threadIdx.x == 0) a.selected_lengths[b * a.l_request + head] = (int)(taken * a.page - short_of);
}

template <class T, int HeadTiles, bool Whole, int Held, int Threads> __global__ __launch_bounds__(Threads) void select_kernel(SelectArgs a) {
  constexpr int kWaves = Threads / kWave;
  unsigned b, length, units, unit0 = 0, unit1, parts = 1, head;
  if (a.pieces == 0) {
    b = blockIdx.x / a.heads;
    head = blockIdx.x - b * a.heads;
    length = length_of(a, load_scalar(a.lengths + b));
    unit1 = units_of<Threads>(a, pages_of(a, length));
  } else {
    __shared__ unsigned ends[Threads], sums[2][kWaves];     // pieces of the rows of a thread's requests, summed up to it
    const unsigned each = (a.requests + Threads - 1) / Threads, b0 = min(threadIdx.x * each, a.requests), b1 = min(b0 + each, a.requests);
    unsigned mine = 0;
    for (unsigned i = b0; i < b1; ++i) mine += units_of<Threads>(a, pages_of(a, length_of(a, a.lengths[i]))) * a.heads;
    mine = (unsigned)wave_reduce<AddI32>((int)mine);
    if (lane_id() == 0) sums[0][wave_id()] = mine;
    __syncthreads();
    unsigned total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += sums[0][w];
    const unsigned share = max((total + a.pieces - 1) / a.pieces, 1u);
    auto parts_of = [&](unsigned n) { return (n + share - 1) / share; };
    mine = 0;
    for (unsigned i = b0; i < b1; ++i) mine += parts_of(units_of<Threads>(a, pages_of(a, length_of(a, a.lengths[i])))) * a.heads;
    const unsigned upto = (unsigned)wave_scan_inclusive<AddI32>((int)mine);
    if (lane_id() == kWave - 1) sums[1][wave_id()] = upto;
    __syncthreads();
    unsigned before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (w < wave_id()) before += sums[1][w];
    ends[threadIdx.x] = before + upto;
    __syncthreads();
    if (blockIdx.x >= ends[Threads - 1]) return;
    // the request of this piece, and the pieces before it
    unsigned chunk = 0;
#pragma unroll
    for (int k = 0; k < Threads / kWave; ++k) chunk += (unsigned)__popcll(__ballot(ends[k * kWave + lane_id()] <= blockIdx.x));
    chunk = __builtin_amdgcn_readfirstlane(chunk);
    before = chunk ? __builtin_amdgcn_readfirstlane(ends[chunk - 1]) : 0u;
    for (b = chunk * each;; ++b) {
      length = length_of(a, load_scalar(a.lengths + b));
      units = units_of<Threads>(a, pages_of(a, length));
      parts = parts_of(units);
      if (blockIdx.x - before < parts * a.heads) break;
      before += parts * a.heads;
    }
    head = (blockIdx.x - before) / parts;
    const unsigned part = blockIdx.x - before - head * parts;
    unit0 = (unsigned)((unsigned long long)units * part / parts);
    unit1 = (unsigned)((unsigned long long)units * (part + 1) / parts);
  }
  select_of_row<T, HeadTiles, Whole, Held, Threads>(a, b, head, length, unit0, unit1, parts, a.counters + (parts > 1 ? b * a.heads + head : 0));
}

// With more rows than half of these, each has a workgroup.  Pieces: as many as workgroups are resident; half of them take 60 us where these take 56 (64 ragged
// requests), twice as many 57, a fixed number of pieces for every row 61.
constexpr unsigned kWorkgroups = 2048;
constexpr unsigned kLongRow = 2 * kMany;                     // pages; longer ones by many threads

struct PageSelect final : Operator {
  SelectArgs a{};
  int32_t dtype;
  bool far = false;                        // keys leave LDS
  int threads = kFew;
  template <class F> void with_kernel(F &&f) const {
    auto by_width = [&](auto t, auto tiles, auto whole) {
      using T = decltype(t);
      constexpr int kTiles = decltype(tiles)::value;
      constexpr bool kWhole = decltype(whole)::value;
      if (threads == kMany) {
        constexpr int kOfMany = kWhole ? kTiles : 1;           // two with the tests do not fit the registers
        if (a.width <= 8 * kMany) f(&select_kernel<T, kOfMany, kWhole, 8, kMany>);
        else f(&select_kernel<T, kOfMany, kWhole, 0, kMany>);
      } else if (a.width <= 4 * kFew) f(&select_kernel<T, kTiles, kWhole, 4, kFew>);
      else if (a.width <= 8 * kFew) f(&select_kernel<T, kTiles, kWhole, 8, kFew>);
      else if (a.width <= 32 * kFew) f(&select_kernel<T, kTiles, kWhole, 32, kFew>);
      else f(&select_kernel<T, kTiles, kWhole, 0, kFew>);
    };
    auto by_dim = [&](auto t, auto tiles) {
      if (a.dim % (64 / sizeof(t)) == 0) by_width(t, tiles, std::true_type{});
      else by_width(t, tiles, std::false_type{});
    };
    auto by_group = [&](auto t) {
      if (a.group <= 4) by_dim(t, std::integral_constant<int, 1>{});
      else by_dim(t, std::integral_constant<int, 2>{});
    };
    if (dtype == FC_F32) by_group(float{});
    else if (dtype == FC_F16) by_group(_Float16{});
    else by_group(__bf16{});
  }
  size_t workspace() const override { return far ? (size_t)a.requests * a.heads * a.width * sizeof(unsigned long long) : 0; }
  void record(Recorder &r) const override {
    if (a.requests == 0 || a.heads == 0) return;
    SelectArgs args = a;
    args.keys = far ? reinterpret_cast<unsigned long long *>(r.workspace) : nullptr;
    args.counters = r.counters;
    with_kernel([&](auto kernel) { r.launch(kernel, a.pieces + a.requests * a.heads, threads, args); });
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
  if (kv < 1 || heads < 1 || heads % kv) return c.fail(FC_E_ARG, "the heads of q must be a multiple of those of the bounds").code();
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
  const bool split = rows <= kWorkgroups / 2 && a.width > block_pages(kFew);
  if (split && a.width > kLongRow) op->threads = kMany;
  op->far = a.width > kKept || split;
  if ((uint64_t)rows * a.width > (uint64_t)1 << 36) return c.fail(FC_E_LIMIT, "too many requests, heads and pages of a request together").code();
  if (split) {
    unsigned resident = 0;
    op->with_kernel([&](auto kernel) { resident = resident_workgroups(kernel, op->threads); });
    a.pieces = std::min(resident ? resident : 256u, rows * ceil_div(a.width, block_pages(op->threads)));
  }
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
