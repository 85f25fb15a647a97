// Attention of requests that share a prefix (include/fc.h, fc_prefix_attention): the keys of the prefix are read once for all of them.
//
// The query heads of all requests of a group that read the same key head are columns of one product, 32 of them a wave; a workgroup has
// `columns` = 32, 64 or 128 (16 where there are no more), its other waves take other keys.  Keys and values of a step go through LDS, which all columns read them from:
//   scores  = K q^T, outputs = V^T p^T, as in attention.hpp: lane (r, g), r = lane % 16, g = lane / 16, has columns r and 16 + r and the
//   keys 4g .. 4g+3 of every 16, in whose order the values' product takes them from LDS.
// What a workgroup has of a row (prefix.hpp) is written as it is: the attention of the requests' own keys, which follows, joins it.
//
// A step of 32 keys (16 of 32 bits) and 32 columns costs a wave 2 * 8 products for the scores and 2 * 16 for the values (128 elements of 16 bits, weights in two
// parts), nine to ten vector instructions for each of its 16 scores a lane, and 16 kB from LDS; the three add up, since all waves of a workgroup come to each of them at about the same time.
// A unit's keys and values are asked for while the one before is worked on, their places two units before.
//
// What bounds it.  One prefix of 32768 keys, 8 key heads of 128, 64 requests of 32 heads (bf16, 134 MB, 34 GFLOP) 76 us: matrix instructions 22 us, vector
// instructions 25, LDS 17, the start and the pieces (38 MB) 11; without the arithmetic 41 to 54.  4096 keys, 4 key heads, 192 requests of 32 heads 42 us.  Five of 1501 to 3001 keys, 6
// heads of 96, 31 requests (f32, 55 MB) 26.5 us: six or seven of 16 columns have a query, and a matrix instruction of 32 bits has an eighth of the products of one of 16
// bits and takes twice as long (32 cycles and 16); two workgroups a compute unit instead of one gain nothing.
// 500 keys, 2 key heads of 64, 4 requests of 8 heads (f16) 6.4 us: the launch, the groups, then pages, keys and products one after the other.
#include "attention.hpp"

#include <algorithm>
#include <cmath>

namespace fc {

extern template AttentionKernel attention_kernel_of<Form::kAfterPrefix>(int32_t, unsigned, bool);

namespace {

struct PrefixArgs {
  const char *q, *k, *v;
  const int *table, *lengths, *start;      // of the groups
  float *pieces;                           // DEVICE
  unsigned *plan;                          // DEVICE
  long long q_request, q_head, table_stride;
  long long k_page, k_place, k_head, v_page, v_place, v_head;
  unsigned long long page_factor;          // n / page = n * page_factor >> page_shift, n below 2^31
  unsigned page_shift;
  unsigned requests, groups, kv_heads, group, dim, page, pages, width, workers;
  float scale;
};

// What the groups come to, in LDS.  Group g has the requests starts[g] .. starts[g+1]-1; its rows are rows[g] .. and its units units[g] ..
// counted over all groups.
struct Plan {
  unsigned starts[kPrefixGroups + 1], rows[kPrefixGroups + 1], units[kPrefixGroups + 1];
};

__device__ __forceinline__ unsigned keys_of_group(const PrefixArgs &a, unsigned g) {
  return a.pages ? (unsigned)min((unsigned long long)max(a.lengths[g], 0), (unsigned long long)a.width * a.page) : 0u;
}

// the largest g below n for which at[g] <= x (at[0] <= x)
__device__ __forceinline__ unsigned last_at_or_below(const unsigned *at, unsigned n, unsigned x) {
  unsigned low = 0;
  while (n > 1) {
    const unsigned half = n / 2;
    if (at[low + half] <= x) { low += half; n -= half; }
    else n = half;
  }
  return low;
}

template <int Columns, int Tile> __device__ __forceinline__ void make_plan(const PrefixArgs &a, Plan &plan) {
  if (wave_id() == 0) {
    // starts that go back, or lie outside the batch, leave empty groups
    int reached = 0;
    unsigned row = 0, unit = 0;
    for (unsigned g0 = 0; g0 <= a.groups; g0 += kWave) {
      const unsigned g = g0 + lane_id();
      const int begin = max(reached, wave_scan_inclusive<MaxI32>(g <= a.groups ? min(max(a.start[g], 0), (int)a.requests) : 0));
      if (g <= a.groups) plan.starts[g] = (unsigned)begin;
      reached = __builtin_amdgcn_readlane(begin, kWave - 1);
    }
    __builtin_amdgcn_wave_barrier();
    for (unsigned g0 = 0; g0 < a.groups; g0 += kWave) {
      const unsigned g = g0 + lane_id();
      unsigned rows = 0, units = 0;
      if (g < a.groups) {
        const unsigned n = plan.starts[g + 1] - plan.starts[g];
        units = n ? ceil_div(keys_of_group(a, g), Tile) : 0u;
        rows = units ? a.kv_heads * ceil_div((unsigned long long)n * a.group, Columns) : 0u;
        units *= rows;
      }
      const unsigned rows_to = (unsigned)wave_scan_inclusive<AddI32>((int)rows), units_to = (unsigned)wave_scan_inclusive<AddI32>((int)units);
      if (g < a.groups) {
        plan.rows[g] = row + rows_to - rows;
        plan.units[g] = unit + units_to - units;
      }
      row += (unsigned)__builtin_amdgcn_readlane((int)rows_to, kWave - 1);
      unit += (unsigned)__builtin_amdgcn_readlane((int)units_to, kWave - 1);
    }
    if (lane_id() == 0) {
      plan.rows[a.groups] = row;
      plan.units[a.groups] = unit;
    }
  }
  __syncthreads();
}

// Where a key and its value lie, in elements from the first of their key head
struct Key {
  long long k, v;
};

// 4 elements of 16 bits in LDS, which 16 lanes change among themselves: lane r gets the r-th of the 16 elements of lanes 0 to 3, of 4 to 7, of 8 to 11
// and of 12 to 15
template <class T> __device__ __forceinline__ Vec<T, 4> read_turned(const T *from) {
  using Raw = Vec<short, 4>;
  return __builtin_bit_cast(Vec<T, 4>, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Raw *)reinterpret_cast<uintptr_t>(from)));
}

// Tiles: of 16 columns of a wave
template <class T, int Dim, int ColumnWaves, int Tiles> struct PrefixShape {
  static constexpr int kTiles = Tiles;
  static constexpr int kColumns = 16 * kTiles * ColumnWaves, kKeyWaves = kWaves / ColumnWaves;
  static constexpr int kSteps = kKeyWaves == 1 ? 2 : 1, kTile = Kind<T>::kKeys * kKeyWaves * kSteps;
  static constexpr int kWide = 16 / sizeof(T), kRow = Dim / kWide;           // 16 bytes of a key; of them in a row
  static constexpr int kLoads = kTile * kRow / kThreads;                     // of K, and of V, of a thread
  // 16 bits: 32 bytes between the values of two keys, so that the four rows that a turned read takes start at different banks
  static constexpr int kValueRow = Dim + (sizeof(T) == 2 ? 16 : 0);
  static constexpr size_t kTileBytes = (size_t)kTile * (Dim + kValueRow) * sizeof(T);
  static constexpr size_t kJoinBytes = (size_t)(kWaves - ColumnWaves) * (kTiles * Dim / 4 + 4) * kWave * sizeof(float);
  static constexpr size_t kRowsBytes = (size_t)ColumnWaves * 16 * (Dim + 4) * sizeof(float);
  static constexpr size_t kBytes = std::max({kTileBytes, kJoinBytes, kRowsBytes});
};

// where 16 bytes of a key's row lie in LDS: rows that are read side by side start at different banks
template <int Row> __device__ __forceinline__ unsigned place_in_lds(unsigned key, unsigned chunk) {
  const unsigned turn = Row >= 16 ? key & 15 : (key >> 1) & 7;
  return key * Row + (chunk ^ turn);
}

template <class T, int Dim, int ColumnWaves, int Tiles>
__global__ __launch_bounds__(kThreads, Dim == 256 || (Dim == 128 && Tiles == 2 && (ColumnWaves == 1 || sizeof(T) == 4)) ? 1 : 2) void prefix_kernel(PrefixArgs a) {
  using S = PrefixShape<T, Dim, ColumnWaves, Tiles>;
  constexpr int kKeys = Kind<T>::kKeys, kSub = kKeys / 16, kWide = S::kWide, kChunks = Dim / (4 * kWide), kRow = S::kRow;
  constexpr int kW = Dim / 16, kParts = kW < kWide ? 1 : kW / kWide, kPart = kW < kWide ? kW : kWide;
  constexpr int kTiles = S::kTiles;
  // weights of f16, 2^14 larger than they are, end at 2^16.  0, every new maximum at once: 8 groups of 128 columns, 4096 keys, 8 key heads of 128 63 us
  // and 60 this way (bf16), 210 and 196 (f32), 4 groups of 64 columns 73 and 68 (f32).
  constexpr float kSlack = sizeof(T) == 4 ? 5.0f : Kind<T>::kShift ? 1.0f : 8.0f;
  using Frag = Vec<T, kWide>;
  using Part = Vec<T, kPart>;
  __shared__ Plan plan;
  __shared__ __attribute__((aligned(16))) char bytes[S::kBytes];
  __shared__ Key keys[4][S::kTile];
  __shared__ unsigned long long there[4][2];
  make_plan<S::kColumns, S::kTile>(a, plan);
  const unsigned total = plan.units[a.groups], share = max((total + a.workers - 1) / a.workers, 1u);
  // what the others do is written down for the launch that joins it, some requests by each
  if (blockIdx.x == 0 && threadIdx.x == 0) a.plan[0] = share;
  for (unsigned b = blockIdx.x * kThreads + threadIdx.x; b < a.requests; b += a.workers * kThreads) {
    unsigned words[5] = {};
    if (b >= plan.starts[0] && b < plan.starts[a.groups]) {
      const unsigned g = last_at_or_below(plan.starts, a.groups, b), n = plan.starts[g + 1] - plan.starts[g];
      const unsigned rows = plan.rows[g + 1] - plan.rows[g];
      words[0] = plan.units[g];
      words[1] = rows ? (plan.units[g + 1] - plan.units[g]) / rows : 0u;
      words[2] = b - plan.starts[g];
      words[3] = ceil_div((unsigned long long)n * a.group, S::kColumns);
      words[4] = plan.rows[g];
    }
#pragma unroll
    for (int i = 0; i < 5; ++i) a.plan[8 + 8 * (size_t)b + i] = words[i];
  }
  Frag *const lds_k = reinterpret_cast<Frag *>(bytes);
  T *const lds_v = reinterpret_cast<T *>(bytes) + S::kTile * Dim;
  const unsigned r = lane_id() & 15, g4 = lane_id() >> 4;
  const unsigned wave = uniform((unsigned)wave_id()), column_wave = wave % ColumnWaves, key_wave = wave / ColumnWaves;
  const T *const q0 = reinterpret_cast<const T *>(a.q);
  // 16 bits: m is half a product of q and k until the piece is written, and `by` takes differences of such halves to powers of 2.  A difference is taken
  // first, so that the largest key's is 0 whatever its product is: the rounding of a large product times `by` would be many powers of 2.  The
  // difference of two products need not be a finite number of 32 bits where its power of 2 is; that of their halves is one.  An instruction a score more than
  // products times `by` less the maximum's: 64 requests behind 32768 keys 125.7 us and 124.1.
  constexpr float kOfProduct = sizeof(T) == 4 ? 1.0f : 0.5f;
  const float by = sizeof(T) == 4 ? 1.0f : a.scale == 0.0f ? 1.0f : fabsf(a.scale) * (kLog2e / kOfProduct);
  auto power = [by](float x) { return sizeof(T) == 4 ? exp_of(x) : __builtin_amdgcn_exp2f(x * by); };
  unsigned at = (unsigned)min((unsigned long long)blockIdx.x * share, (unsigned long long)total);
  const unsigned end = min(at + share, total);
  while (at < end) {
    const unsigned g = uniform(last_at_or_below(plan.units, a.groups, at));
    const unsigned members = plan.starts[g + 1] - plan.starts[g], blocks = ceil_div((unsigned long long)members * a.group, S::kColumns);
    const unsigned length = uniform(keys_of_group(a, g)), units = ceil_div(length, S::kTile);
    const unsigned row = uniform((at - plan.units[g]) / units), unit0 = at - plan.units[g] - row * units, unit1 = min(units, unit0 + (end - at));
    const unsigned kv = row / blocks, column0 = (row - kv * blocks) * S::kColumns + column_wave * 16 * kTiles;
    const unsigned columns = members * a.group;
    const int *const table = a.table + g * a.table_stride;
    const unsigned chunk = threadIdx.x % kRow, key0 = threadIdx.x / kRow;
    const T *const k0 = reinterpret_cast<const T *>(a.k) + kv * a.k_head + min(chunk * kWide, a.dim - kWide);
    const T *const v0 = reinterpret_cast<const T *>(a.v) + kv * a.v_head + min(chunk * kWide, a.dim - kWide);
    Frag q[kTiles][kChunks];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const unsigned column = column0 + 16 * t + r;
      const unsigned member = min(column, columns - 1) / a.group, head = min(column, columns - 1) - member * a.group;
      const T *from = q0 + (plan.starts[g] + member) * a.q_request + (kv * a.group + head) * a.q_head;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const unsigned d = (c * 4 + g4) * kWide;
        Frag f;
#pragma unroll
        for (int i = 0; i < kWide; ++i) f[i] = (T)0.0f;
        if (column < columns && d < a.dim) f = load_vec<T, kWide>(from + d);
        if constexpr (sizeof(T) == 2)                        // scores are then multiplied by a number above 0
          if (!(a.scale > 0.0f))
#pragma unroll
            for (int i = 0; i < kWide; ++i) f[i] = a.scale < 0.0f ? -f[i] : f[i] * (T)0.0f;
        q[t][c] = f;
      }
    }
    Acc o[kTiles][kW];
    float m[kTiles], l[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      m[t] = -__builtin_inff();
      l[t] = 0.0f;
#pragma unroll
      for (int j = 0; j < kW; ++j) o[t][j] = Acc{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // where the keys of a unit lie, a thread for each: its page is asked for a unit before it is written down
    const bool looks = threadIdx.x < (unsigned)((S::kTile + kWave - 1) / kWave * kWave);
    auto page_of = [&](unsigned unit) {
      const unsigned j = unit * S::kTile + threadIdx.x;
      const bool mine = threadIdx.x < (unsigned)S::kTile && unit < unit1 && j < length;
      return mine ? (unsigned)table[(unsigned)((unsigned long long)j * a.page_factor >> a.page_shift)] : a.pages;
    };
    auto write_down = [&](unsigned unit, unsigned page) {
      const unsigned j = unit * S::kTile + threadIdx.x, w = (unsigned)((unsigned long long)j * a.page_factor >> a.page_shift);
      const unsigned long long mask = __ballot(page < a.pages);
      // a key that is not there is read where the first page's first lies
      if (threadIdx.x < (unsigned)S::kTile) keys[unit & 3][threadIdx.x] = page < a.pages ? Key{page * a.k_page + (j - w * a.page) * a.k_place, page * a.v_page + (j - w * a.page) * a.v_place} : Key{0, 0};
      if (lane_id() == 0) there[unit & 3][wave] = mask;
    };
    Frag next_k[S::kLoads], next_v[S::kLoads];
    auto load = [&](unsigned unit) {
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i) {
        const Key key = keys[unit & 3][key0 + i * (kThreads / kRow)];
        next_k[i] = load_vec<T, kWide>(k0 + key.k);
        next_v[i] = load_vec<T, kWide>(v0 + key.v);
      }
    };
    // whether all keys of a unit are there
    auto is_whole = [&](unsigned unit) {
      return there[unit & 3][0] == (S::kTile >= 64 ? ~0ull : (1ull << S::kTile % 64) - 1) && (S::kTile <= 64 || there[unit & 3][1] == ~0ull);
    };
    __syncthreads();                                         // the row before is done with LDS
    unsigned page = a.pages;
    if (looks) {
      const unsigned first = page_of(unit0), second = page_of(unit0 + 1);
      page = page_of(unit0 + 2);
      write_down(unit0, first);
      write_down(unit0 + 1, second);
    }
    __syncthreads();
    load(unit0);
    for (unsigned unit = unit0; unit < unit1; ++unit) {
      __syncthreads();                                       // the unit before is read
      if (a.dim < (unsigned)Dim && chunk * kWide >= a.dim)   // past the end of a head, whose query is zero there
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i)
#pragma unroll
          for (int e = 0; e < kWide; ++e) next_k[i][e] = (T)0.0f;
      if (!is_whole(unit))                                   // the weight of a key that is not there is zero, its value must not be more
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) {
          const unsigned key = key0 + i * (kThreads / kRow);
          const bool mine = there[unit & 3][key / 64] >> key % 64 & 1;
#pragma unroll
          for (int e = 0; e < kWide; ++e) next_v[i][e] = mine ? next_v[i][e] : (T)0.0f;
        }
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i) {
        const unsigned key = key0 + i * (kThreads / kRow);
        lds_k[place_in_lds<kRow>(key, chunk)] = next_k[i];
        store_vec<T, kWide>(lds_v + key * S::kValueRow + chunk * kWide, next_v[i]);
      }
      if (looks) write_down(unit + 2, page);
      __syncthreads();
      load(unit + 1 < unit1 ? unit + 1 : unit);
      if (looks) page = page_of(unit + 3);
#pragma clang loop unroll_count(Dim == 256 ? 1 : S::kSteps)
      for (int step = 0; step < S::kSteps; ++step) {
        const unsigned first = (key_wave * S::kSteps + step) * kKeys;
        const unsigned live = (unsigned)(there[unit & 3][first / 64] >> first % 64) & (kKeys == 32 ? 0xffffffffu : 0xffffu);
        float p[kTiles][kSub][4];
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
          constexpr int kSums = sizeof(T) == 4 ? 4 : 1;
          Acc part[kTiles][kSums];
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int n = 0; n < kSums; ++n) part[t][n] = Acc{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const Frag k = lds_k[place_in_lds<kRow>(first + 16 * u + r, c * 4 + g4)];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) part[t][c % kSums] = mma(k, q[t][c], part[t][c % kSums]);
            if (Dim == 256 && c % 2 == 1) __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            Acc score = part[t][0];
            if constexpr (kSums == 4) score = ((part[t][0] + part[t][1]) + (part[t][2] + part[t][3])) * a.scale;
#pragma unroll
            for (int i = 0; i < 4; ++i) p[t][u][i] = score[i];
          }
        }
        if (live != (kKeys == 32 ? 0xffffffffu : 0xffffu)) {
#pragma unroll
          for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!(live >> (16 * u + 4 * g4 + i) & 1))
#pragma unroll
                for (int t = 0; t < kTiles; ++t) p[t][u][i] = -__builtin_inff();
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          float most = -__builtin_inff();
#pragma unroll
          for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, p[t][u][i]);
          // m may stay behind the largest score by kSlack, so that sums are seldom multiplied
          most *= kOfProduct;
          if (__any((most - m[t]) * by > kSlack)) {
            most = fmaxf(column_max(most), m[t]);
            const float keep = most == -__builtin_inff() ? 1.0f : power(m[t] - most);
            m[t] = most;
            l[t] *= keep;
#pragma unroll
            for (int j = 0; j < kW; ++j) o[t][j] *= keep;
          }
          const float top = m[t] == -__builtin_inff() ? 0.0f : m[t];
#pragma unroll
          for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              p[t][u][i] = sizeof(T) == 2 ? __builtin_amdgcn_exp2f(fmaf(fmaf(p[t][u][i], kOfProduct, -top), by, (float)Kind<T>::kShift)) : exp_of(p[t][u][i] - top);
              l[t] += p[t][u][i];
            }
        }
        if constexpr (sizeof(T) == 2) {
          Vec<T, 8> high[kTiles], low[kTiles];
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              T upper, rest;
              split(p[t][e / 4][e % 4], upper, rest);
              high[t][e] = upper;
              low[t][e] = rest;
            }
          // a read gives each lane r the element 16 j + r of the keys 4g .. 4g+3: it takes four elements of key 4g + r / 4 and has them change lanes
          const T *const from = lds_v + (first + 4 * g4 + r / 4) * S::kValueRow + r % 4 * 4;
#pragma unroll
          for (int j = 0; j < kW; ++j) {
            const Vec<T, 8> values = __builtin_shufflevector(read_turned(from + 16 * j), read_turned(from + 16 * S::kValueRow + 16 * j), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
              o[t][j] = mma(values, high[t], o[t][j]);
              o[t][j] = mma(values, low[t], o[t][j]);
            }
            if (Dim == 256 && j % 2 == 1) __builtin_amdgcn_sched_barrier(0);   // no further reads ahead: registers
          }
        } else {
          Part vf[4][kParts];
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < kParts; ++n) vf[i][n] = load_vec<T, kPart>(lds_v + (first + 4 * g4 + i) * S::kValueRow + (16 * n + r) * kPart);
#pragma unroll
          for (int j = 0; j < kW; ++j)
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
              o[t][j] = mma(Vec<float, 4>{vf[0][j / kPart][j % kPart], vf[1][j / kPart][j % kPart], vf[2][j / kPart][j % kPart], vf[3][j / kPart][j % kPart]},
                            Vec<float, 4>{p[t][0][0], p[t][0][1], p[t][0][2], p[t][0][3]}, o[t][j]);
        }
      }
    }
    // the waves of other keys hand theirs to the first of these columns, lane by lane
    if constexpr (S::kKeyWaves > 1) {
      constexpr int kValues = kTiles * kW * 4 + 4;
      float *const shared = reinterpret_cast<float *>(bytes);
      auto slot = [&](unsigned w, int value) { return shared + ((size_t)((w - ColumnWaves) * kValues + value)) * kWave + lane_id(); };
      __syncthreads();                                       // the last unit is read
      if (key_wave > 0) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          *slot(wave, 2 * t) = m[t];
          *slot(wave, 2 * t + 1) = l[t];
#pragma unroll
          for (int j = 0; j < kW; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) *slot(wave, 4 + (t * kW + j) * 4 + i) = o[t][j][i];
        }
      }
      __syncthreads();
      if (key_wave == 0)
        for (unsigned w = wave + ColumnWaves; w < (unsigned)kWaves; w += ColumnWaves)
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            const float other = *slot(w, 2 * t), most = fmaxf(m[t], other), base = most == -__builtin_inff() ? 0.0f : most;
            const float keep = power(m[t] - base), f = power(other - base);
            m[t] = most;
            l[t] = l[t] * keep + *slot(w, 2 * t + 1) * f;
#pragma unroll
            for (int j = 0; j < kW; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[t][j][i] = o[t][j][i] * keep + *slot(w, 4 + (t * kW + j) * 4 + i) * f;
          }
    }
    // A lane's sums lie 16 bytes here and there in a piece; they pass through LDS, a tile of 16 columns at a time, so that a wave writes rows.
    __syncthreads();                                         // all are done with LDS
    if (key_wave == 0) {
      const size_t floats = prefix_piece_floats(S::kColumns, a.dim);
      float *const piece = a.pieces + (size_t)(blockIdx.x + plan.rows[g] + row) * floats, *const rows = reinterpret_cast<float *>(bytes) + wave * 16 * (Dim + 4);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const unsigned first = column_wave * 16 * kTiles + 16 * t, live = min(columns - min(columns, column0 + 16 * t), 16u);
        const float sum = column_sum(l[t]);
        if (live == 0) continue;
        float *const mine = rows + r * (Dim + 4);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int j = 0; j < kW; ++j) store_vec<float, 4>(mine + 16 * j + 4 * g4, o[t][j]);
        } else {
#pragma unroll
          for (int n = 0; n < kParts; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              store_vec<float, 4>(mine + (n * 16 + 4 * g4 + i) * kPart, Vec<float, 4>{o[t][n * kPart][i], o[t][n * kPart + 1][i], o[t][n * kPart + 2][i], o[t][n * kPart + 3][i]});
        }
        __builtin_amdgcn_wave_barrier();
        for (unsigned x = lane_id(); x < live * (Dim / 4); x += kWave) {
          const unsigned column = x / (Dim / 4), d = x % (Dim / 4) * 4;
          if (d < a.dim) store_vec<float, 4>(piece + (size_t)(first + column) * a.dim + d, *reinterpret_cast<const Vec<float, 4> *>(rows + column * (Dim + 4) + d));
        }
        __builtin_amdgcn_wave_barrier();
        const float top = sizeof(T) == 4 || m[t] == -__builtin_inff() ? m[t] : m[t] * (fabsf(a.scale) / kOfProduct);          // a score, rounded as in attention.hpp
        if (g4 == 0 && r < live) store_vec<float, 2>(piece + (size_t)S::kColumns * a.dim + 2 * (first + r), Vec<float, 2>{top, sum});
      }
    }
    at += unit1 - unit0;
  }
}

using PrefixKernel = void (*)(PrefixArgs);
struct Variant {
  PrefixKernel kernel;
  unsigned columns, tile;
};
template <class T, int Dim, int ColumnWaves, int Tiles> Variant variant() {
  using S = PrefixShape<T, Dim, ColumnWaves, Tiles>;
  return {&prefix_kernel<T, Dim, ColumnWaves, Tiles>, (unsigned)S::kColumns, (unsigned)S::kTile};
}
// As many columns as groups have on average: what is left empty costs as much as what is not, and more columns read the prefix less often.  16 instead of 32:
// 6 requests of a head a key head (f32) 26.5 us and 35, 4 of four (f16) 6.4 and 7.5.  Groups of 4096 keys, 8 key heads of 128, us with 32 / 64 / 128 columns:
//   8 of 32 columns 42 / 40 / 50 (bf16), 81 / 113 / 179 (f32);  8 of 64 63 / 43 / 51, 143 / 117 / 183;  8 of 128 108 / 68 / 60, 266 / 220 / 195
// The average is over all requests and all places for groups, since which of them are in use is only known on the device.  Where most requests have no group it is too
// large: one prefix of 4096 keys, 8 readers of four heads a key head, 38 us where they are the batch and 56 among 256 requests, whose rows are written too (bf16), 43.5 and 51.5 (f32).  Where
// most places hold no group it is too small: 64 readers, 1 / 4 / 16 / 64 places 44.5 / 34 / 47 / 47 us (bf16), 65 / 67 / 94 / 94 (f32).
// Heads of more than 128 elements of 16 bits have 128 columns however few are in use.  One group, 4096 keys, 8 key heads of 256 (bf16), us with 128 / 64 / 32 / 16 columns:
//   16 in use 63 / 60 / 59 / 62;  32 65 / 61 / 60 / 46;  64 66 / 62 / 46 / 44;  128 68 / 50 / 46 / 57
template <class T, int Dim> Variant variant_of_heads(unsigned columns) {
  constexpr int kMost = sizeof(T) == 4 && Dim == 256 ? 1 : 2;                  // tiles that the registers hold
  if constexpr (Dim < 256) {
    if (columns <= 16) return variant<T, Dim, 1, 1>();
    if (columns <= 32) return variant<T, Dim, 1, kMost>();
  }
  if constexpr (Dim < 256 || sizeof(T) == 4)
    if (columns <= 32 * kMost) return variant<T, Dim, 2, kMost>();
  return variant<T, Dim, 4, kMost>();
}
template <class T> Variant variant_of_type(unsigned dim, unsigned columns) {
  return dim <= 64 ? variant_of_heads<T, 64>(columns) : dim <= 128 ? variant_of_heads<T, 128>(columns) : variant_of_heads<T, 256>(columns);
}

size_t whole_lines(size_t bytes) { return (bytes + 255) / 256 * 256; }

struct PrefixAttention final : Operator {
  Attention own;
  PrefixArgs a{};
  Variant variant{};
  unsigned most_rows = 0, most_units = 0;
  bool any_prefix = false;
  size_t plan_bytes() const { return whole_lines(PrefixPlan::bytes(a.requests)); }
  size_t pieces_bytes() const { return whole_lines(((size_t)a.workers + most_rows) * prefix_piece_floats(variant.columns, a.dim) * sizeof(float)); }
  size_t workspace() const override { return any_prefix ? plan_bytes() + pieces_bytes() + own.workspace() : own.workspace(); }
  void record(Recorder &r) const override {
    if (own.a.requests == 0 || own.a.group == 0) return;
    if (!any_prefix) return own.record(r);
    PrefixArgs args = a;
    args.plan = reinterpret_cast<unsigned *>(r.workspace);
    args.pieces = reinterpret_cast<float *>(r.workspace + plan_bytes());
    r.launch(variant.kernel, a.workers, kThreads, args);
    Recorder behind{r.launches, r.workspace + plan_bytes() + pieces_bytes(), r.counters, r.what};
    Attention after = own;
    after.a.prefix_plan = args.plan;
    after.a.prefix_pieces = args.pieces;
    after.a.prefix_columns = variant.columns;
    after.record(behind);
  }
  const char *name() const override { return "prefix attention"; }
};

}  // namespace

int make_prefix_attention(const fc_prefix_attention &n, std::unique_ptr<Operator> &out, std::string &err) {
  auto op = std::make_unique<PrefixAttention>();
  fc_paged_attention own{};
  own.q = n.q;
  own.k_cache = n.k_cache;
  own.v_cache = n.v_cache;
  own.table = n.table;
  own.lengths = n.lengths;
  own.out = n.out;
  own.lse = n.lse;
  own.scale = n.scale;
  TensorChecks c(err);
  c.array("prefix_table", n.prefix_table, FC_I32, {-1, -1});
  const int64_t groups = n.prefix_table.shape[0];
  c.array("prefix_lengths", n.prefix_lengths, FC_I32, {groups});
  c.array("group_start", n.group_start, FC_I32, {groups + 1});
  if (!c.ok()) return c.code();
  if (groups > kPrefixGroups) return c.fail(FC_E_LIMIT, "more than " + std::to_string(kPrefixGroups) + " groups").code();
  const uint64_t keys = std::min<uint64_t>((uint64_t)n.prefix_table.shape[1] * (uint64_t)std::max<int64_t>(n.k_cache.shape[1], 0), 0x7fffffffu);
  op->any_prefix = groups > 0 && keys > 0 && n.k_cache.rank == 4 && n.k_cache.shape[0] > 0;
  op->own.form = op->any_prefix ? Form::kAfterPrefix : Form::kPlain;
  if (const int rc = settle_attention(own, op->own, err); rc != FC_OK) return rc;
  // whose logarithm's base could not be changed in 32 bits
  if (std::fabs(n.scale) >= 0x1p126) return c.fail(FC_E_UNSUPPORTED, "scale must be below 2^126").code();
  const AttentionArgs &o = op->own.a;
  if (op->any_prefix && o.requests && o.group) {
    PrefixArgs &a = op->a;
    a.q = o.q;
    a.k = o.k;
    a.v = o.v;
    a.table = static_cast<const int *>(n.prefix_table.ptr);
    a.lengths = static_cast<const int *>(n.prefix_lengths.ptr);
    a.start = static_cast<const int *>(n.group_start.ptr);
    a.q_request = o.q_request;
    a.q_head = o.q_head;
    a.table_stride = n.prefix_table.stride[0];
    a.k_page = o.k_page;
    a.k_place = o.k_place;
    a.k_head = o.k_head;
    a.v_page = o.v_page;
    a.v_place = o.v_place;
    a.v_head = o.v_head;
    a.requests = o.requests;
    a.groups = (unsigned)groups;
    a.kv_heads = o.kv_heads;
    a.group = o.group;
    a.dim = o.dim;
    a.page = o.page;
    a.pages = o.pages;
    a.width = (unsigned)n.prefix_table.shape[1];
    a.scale = o.scale;
    // factor = ceil(2^(32 + s) / d), 2^s <= d < 2^(s + 1): its error times n is below 2^(32 + s) for n below 2^31, and the product below 2^64
    const unsigned s = 31u - (unsigned)__builtin_clz(a.page);
    a.page_shift = 32 + s;
    a.page_factor = ((1ull << a.page_shift) + a.page - 1) / a.page;
    // columns of a group on average, as many as the waves of a workgroup share where the groups are that large
    const uint64_t columns = (uint64_t)a.requests * a.group;
    const unsigned average = (unsigned)std::min<uint64_t>((columns + groups - 1) / groups, 1u << 20);
    op->variant = op->own.dtype == FC_F32 ? variant_of_type<float>(a.dim, average)
                  : op->own.dtype == FC_F16 ? variant_of_type<_Float16>(a.dim, average) : variant_of_type<__bf16>(a.dim, average);
    // a row for each key head and each `columns` of a group: groups and all columns together
    const uint64_t blocks = std::min<uint64_t>(groups, a.requests) + columns / op->variant.columns;
    const unsigned units = ceil_div(keys, op->variant.tile);
    unsigned rows;
    if (columns > 0x7fffffff || blocks > 0x7fffffff || __builtin_mul_overflow((unsigned)blocks, a.kv_heads, &rows) || __builtin_mul_overflow(rows, units, &op->most_units) ||
        op->most_units > 0x7fffffffu)
      return c.fail(FC_E_LIMIT, "too many requests, heads and pages of a prefix together").code();
    op->most_rows = rows;
    const unsigned resident = resident_workgroups(op->variant.kernel, kThreads);
    a.workers = std::max(1u, std::min(resident ? resident : 256u, op->most_units));
  }
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
