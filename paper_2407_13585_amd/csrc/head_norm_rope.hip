// Norm of query and key heads with the rotation by position in the same pass, into tensors or into the cache, and its gradient
// (include/fc.h, fc_head_norm_rope).
//
// One head of one token is a row of D elements.  2^log2 neighbouring lanes hold a row, each of them two packs of V elements that hold the
// elements of its pairs: (y[i], y[i + R/2]) lie in packs that are R/2 apart, (y[2i], y[2i+1]) side by side in one; behind the rotated part
// and for pairs side by side the packs are half of what there is apart.  So nothing is exchanged between lanes but the sum of
// squares, and the row is read once and written once.  A wave takes one token after the other with some of its heads, so that
// the token's cosines and sines and the weights are read once and stay in registers.  Memory bounds it where it is large, the launch and a chain
// of reads (position, angles, result) where it is small:
//   16384 tokens of 40 heads of 128 (bf16, 338 MB) 60.0 to 60.7 us, 5.6 TB/s; 8192 tokens of 28 (f32, 237 MB) 44.8 us, 5.3 TB/s; 5003 tokens of 16 heads
//   of 80 with three axes (f16, 27 MB) 10.0 to 10.3 us; 64 tokens into the cache 4.7 to 6.0 us; the gradient of the first (505 MB) with the sum
//   of the weights' gradients 92 to 96 us, 5.3 to 5.5 TB/s, of 1237 tokens of 12 heads of 64 (f32, 11.6 MB) 10.4 us, a third of them the second launch.
// Rows that do not fill their lanes are bound by instructions: 12844 tokens of 28 heads (bf16) of 72, 80, 96 and 112 elements, turned as a whole or (112)
// a quarter, 28.9, 30.5, 35.1 and 41.9 us (3.6 to 4.0 TB/s), a quarter of 72 or 80 turned 37.7; their gradients 45.3, 54.1, 57.0 and 69.7,
// a quarter turned 57.3 and 65.7 (2.6 to 3.7 TB/s).
#include "operators.hpp"

#include <algorithm>
#include <cmath>

namespace fc {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr unsigned kMostDim = 512;

struct Rows {                       // [T, heads, D]
  char *ptr;
  long long token, head;            // strides in elements
};

struct HeadsArgs {
  Rows q, k, v, q_out, k_out;       // k_out: the tensor, or place 0 of the cache's pages (head: its stride)
  char *v_cache;
  const void *weight[2];            // of q and of k; NULL: no norm
  const float *cos_sin;             // may be NULL where it has no rows
  const int *positions, *axis_of;
  const long long *slots;           // NULL: keys go to the tensor
  long long angle_stride, position_stride;
  long long k_page, k_place, v_page, v_place, v_head;     // strides of the caches
  unsigned tokens, heads[3];        // of q, k, v
  unsigned dim, half, page, places; // half: R / 2, 0: no rotation; places: of the cache
  unsigned axes, angles;            // rows of positions and of cos_sin
  unsigned lanes_log2, per_wave;    // lanes of a row; heads of a token that a wave takes
  float eps;
  bool wide_angles;                 // rows of cos_sin are aligned for packs
};

// Which elements are turned together, and how a lane comes by both.  kHalves: y[i] and y[i + R/2], in two packs that are R/2 apart.  kNeighbours:
// y[2i] and y[2i+1], side by side in a pack.  kCrossed: y[i] and y[i + R/2] where R/2 is no multiple of a pack: the packs lie as those of neighbours
// do, and the row's turned elements are exchanged through LDS.
constexpr int kHalves = 0, kNeighbours = 1, kCrossed = 2;

// Where a lane's two packs of a row lie, the same for all rows, and which pairs they hold.  The packs of neighbouring lanes lie side by side, so that
// an instruction reads whole lines (6966 tokens of 16 heads of 256, f32, half of them turned, neighbours paired, 46 us; 55 with a lane's two packs in a row).
template <int V, int Pairs> struct Place {
  // the i-th pair is of pack i / kOfPack; one element a pack is half a pair
  static constexpr bool kOwn = Pairs == kNeighbours && V > 1;        // the packs have pairs of their own
  static constexpr int kOfPack = kOwn ? V / 2 : V;
  static constexpr int kAngles = kOfPack < 4 ? kOfPack : 4;          // angles that are read at once
  unsigned at[2];
  // turned: of the pairs, which are those of both packs (kHalves), of one or the other (kOwn; a pack may hold the last turned one and the first that
  // is not), or of the elements (kCrossed)
  bool any, turned[Pairs == kCrossed ? 2 * V : kOwn ? V : 1];
  __device__ __forceinline__ Place(unsigned dim, unsigned half, unsigned chunk) {
    any = 2 * V * chunk < dim;
    const bool in = V * chunk < half;
    if constexpr (Pairs == kCrossed || kOwn) {
      at[0] = V * chunk;
      at[1] = dim / 2 + V * chunk;
    } else {
      at[0] = Pairs == kNeighbours ? 2 * chunk : in ? V * chunk : half + V * chunk;
      at[1] = Pairs == kNeighbours ? 2 * chunk + 1 : in ? half + V * chunk : dim / 2 + V * chunk;
    }
    if constexpr (Pairs == kCrossed) {
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) turned[i] = any && at[i / V] + i % V < 2 * half;
    } else if constexpr (kOwn) {
#pragma unroll
      for (int i = 0; i < V; ++i) turned[i] = at[i / kOfPack] / 2 + i % kOfPack < half;
    } else turned[0] = in;
  }
  __device__ __forceinline__ bool turns(int i) const { return turned[kOwn ? i : 0]; }
  // the pair i in the tables, 0 where it is not turned
  __device__ __forceinline__ unsigned angle(int i) const {
    const unsigned first = Pairs == kNeighbours ? at[kOwn ? i / kOfPack : 0] / 2 : at[0];
    return any && turns(i) ? first + i % kOfPack : 0u;
  }
};

// A lane's part of a row as it lies in memory.
template <class T, int V> struct Packs {
  Vec<T, V> a, b;
};

// zeros where there is nothing, or where `live` is false
template <bool Stream, class T, int V, int Pairs>
__device__ __forceinline__ Packs<T, V> load_packs(const T *row, const Place<V, Pairs> &p, bool live) {
  Packs<T, V> x;
#pragma unroll
  for (int i = 0; i < V; ++i) x.a[i] = x.b[i] = (T)0.0f;
  if (p.any && live) {
    x.a = load_vec<T, V, Stream>(row + p.at[0]);
    x.b = load_vec<T, V, Stream>(row + p.at[1]);
  }
  return x;
}

// its pairs: the i-th is (x[0][i], x[1][i])
template <class T, int V, int Pairs> __device__ __forceinline__ void unpack(const Packs<T, V> &w, const Place<V, Pairs> &, float (&x)[2][V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (Pairs == kNeighbours) {    // a pair lies in a pack, or is the two packs where these are an element each, side by side
      const int e = 2 * i, o = 2 * i + 1;
      x[0][i] = e < V ? (float)w.a[e % V] : (float)w.b[e % V];
      x[1][i] = o < V ? (float)w.a[o % V] : (float)w.b[o % V];
    } else {
      x[0][i] = (float)w.a[i];
      x[1][i] = (float)w.b[i];
    }
  }
}

template <bool Stream, class T, int V, int Pairs>
__device__ __forceinline__ void store_row(T *row, const Place<V, Pairs> &p, const float (&x)[2][V]) {
  if (!p.any) return;
  Vec<T, V> a, b;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (Pairs == kNeighbours) {
      const int e = 2 * i, o = 2 * i + 1;
      if (e < V) a[e % V] = (T)x[0][i]; else b[e % V] = (T)x[0][i];
      if (o < V) a[o % V] = (T)x[1][i]; else b[o % V] = (T)x[1][i];
    } else {
      a[i] = (T)x[0][i];
      b[i] = (T)x[1][i];
    }
  }
  store_vec<T, V, Stream>(row + p.at[0], a);
  store_vec<T, V, Stream>(row + p.at[1], b);
}

// The axes of the pairs lane, lane + 64, .. of a row, a byte each; 255: none.
__device__ __forceinline__ unsigned axes_of_lane(const HeadsArgs &a) {
  if (!a.axis_of) return 0u;
  unsigned axes = ~0u;
#pragma unroll
  for (unsigned k = 0; k < kMostDim / 2 / kWave; ++k)
    if (const unsigned n = lane_id() + kWave * k; n < a.half) axes = (axes & ~(255u << 8 * k)) | min((unsigned)a.axis_of[n], 255u) << 8 * k;
  return axes;
}

// Cosines and sines of the pairs of this lane at token t, not used where nothing is turned: NaN where the tables have no row.  One axis: from the
// one row of the token.
template <int V, int Pairs>
__device__ __forceinline__ void load_angles(const HeadsArgs &a, const Place<V, Pairs> &p, unsigned t, float (&c)[V], float (&s)[V]) {
  if (!a.half) return;
  constexpr int kAngles = Place<V, Pairs>::kAngles;
  const int at = a.axes ? load_scalar(a.positions + t) : -1;
  const bool there = (unsigned)at < a.angles;
  const float *row = a.cos_sin + (there ? at : 0) * a.angle_stride;
  const float none = __builtin_nanf("");
#pragma unroll
  for (int i = 0; i < V; i += kAngles) {
    Vec<float, kAngles> cosines = {}, sines = {};
    if (a.angles) {
      if (a.wide_angles) {
        const float *from = row + p.angle(i);
        cosines = load_vec<float, kAngles>(from);
        sines = load_vec<float, kAngles>(from + a.half);
      } else {
        unsigned first = p.angle(i);
        asm volatile("" : "+v"(first));                      // what follows is not to be kept in registers from token to token
#pragma unroll
        for (int k = 0; k < kAngles; ++k) {
          const unsigned n = Pairs == kNeighbours ? min(first + k, a.half - 1) : first + k;
          cosines[k] = row[n];
          sines[k] = row[a.half + n];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAngles; ++k) {
      c[i + k] = there ? cosines[k] : none;
      s[i + k] = there ? sines[k] : none;
    }
  }
}

// Several axes: the lanes of the wave read a pair each and share them through LDS, as every row of the wave needs the same (5003 tokens of 16 heads
// with three axes 10.9 us; 14.0 where each lane read its pairs from all rows), and take them from there for each row, which frees their
// registers.  shared: kMostDim floats of the wave; kCrossed, where they are put down for each element, the sines with their sign: twice as many.
template <int Pairs> __device__ __forceinline__ void stage_angles(const HeadsArgs &a, unsigned axes, unsigned t, float *shared) {
  __builtin_amdgcn_wave_barrier();                           // the lanes of a wave go together: the token before is done
#pragma unroll
  for (unsigned k = 0; k < kMostDim / 2 / kWave; ++k) {
    const unsigned n = lane_id() + kWave * k, axis = axes >> 8 * k & 255u;
    if (n >= a.half) break;
    const int at = axis < a.axes ? a.positions[axis * a.position_stride + t] : -1;
    float cosine = __builtin_nanf(""), sine = cosine;
    if ((unsigned)at < a.angles) {
      const float *row = a.cos_sin + at * a.angle_stride + n;
      cosine = row[0];
      sine = row[a.half];
    }
    shared[n] = cosine;
    if constexpr (Pairs == kCrossed) {
      shared[a.half + n] = cosine;
      shared[kMostDim + n] = -sine;
      shared[kMostDim + a.half + n] = sine;
    } else shared[kMostDim / 2 + n] = sine;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
template <int V, int Pairs> __device__ __forceinline__ void staged_angles(const Place<V, Pairs> &p, const float *shared, float (&c)[V], float (&s)[V]) {
  constexpr int kAngles = Place<V, Pairs>::kAngles;
  typedef Vec<float, kAngles> Some;
#pragma unroll
  for (int i = 0; i < V; i += kAngles) {
    unsigned at = p.angle(i);
    asm volatile("" : "+v"(at));                             // read for each row: kept, they would take the registers that this is to free
    const float *from = shared + at;
    const Some cosines = *reinterpret_cast<const Some *>(from), sines = *reinterpret_cast<const Some *>(from + kMostDim / 2);
#pragma unroll
    for (int k = 0; k < kAngles; ++k) {
      c[i + k] = cosines[k];
      s[i + k] = sines[k];
    }
  }
}

// kCrossed: y turned by the staged angles, or back (Back).  lds: the row's 2 V floats a lane, where every turned element is put down in its
// partner's place.
template <bool Back, int V> __device__ __forceinline__ void turn_crossed(const Place<V, kCrossed> &p, unsigned half, const float *shared, float *lds, float (&y)[2][V]) {
  constexpr int N = V < 4 ? V : 4;
  typedef Vec<float, N> Some;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (!p.turned[k * V]) continue;
    unsigned at = p.at[k];
    asm volatile("" : "+v"(at));                             // places are not to be kept in registers
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (p.turned[k * V + i]) lds[at + i < half ? at + i + half : at + i - half] = y[k][i];
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (!p.turned[k * V]) continue;
    unsigned at = p.at[k];
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int i = 0; i < V; i += N) {
      const Some other = *reinterpret_cast<const Some *>(lds + at + i), cosines = *reinterpret_cast<const Some *>(shared + at + i),
                 sines = *reinterpret_cast<const Some *>(shared + kMostDim + at + i);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float turned = y[k][i + e] * cosines[e] + other[e] * (Back ? -sines[e] : sines[e]);
        y[k][i + e] = p.turned[k * V + i + e] ? turned : y[k][i + e];
      }
    }
  }
  __builtin_amdgcn_wave_barrier();                           // the next row is put down after this one is read
}

// by value: a choice between two places would put both into memory
template <class T, int V> __device__ __forceinline__ Packs<T, V> either(bool first, const Packs<T, V> &x, const Packs<T, V> &y) {
  Packs<T, V> w;
  w.a = first ? x.a : y.a;
  w.b = first ? x.b : y.b;
  return w;
}
__device__ __forceinline__ Rows either(bool first, Rows a, Rows b) {
  return {first ? a.ptr : b.ptr, first ? a.token : b.token, first ? a.head : b.head};
}
template <class T> __device__ __forceinline__ T *row_of(Rows rows, unsigned t, unsigned head) {
  return reinterpret_cast<T *>(rows.ptr) + t * rows.token + head * rows.head;
}

// ones where there is no weight
template <class T, int V, int Pairs> __device__ __forceinline__ Packs<T, V> load_weight(const void *weight, const Place<V, Pairs> &p) {
  Packs<T, V> w = load_packs<false>(static_cast<const T *>(weight), p, weight != nullptr);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    w.a[i] = weight ? w.a[i] : (T)1.0f;
    w.b[i] = weight ? w.b[i] : (T)1.0f;
  }
  return w;
}

// What a wave does: the heads [first, end) of the tokens blockIdx.x * kWaves + wave, .. ; q, k and v heads are numbered in one row.  A row is
// read while the one before is worked on.
struct Turn {
  bool live, is_q, is_v;
  unsigned head;
  __device__ __forceinline__ Turn(const HeadsArgs &a, unsigned h, unsigned end)
      : live(h < end), is_q(h < a.heads[0]), is_v(h >= a.heads[0] + a.heads[1]), head(is_q ? h : is_v ? h - a.heads[0] - a.heads[1] : h - a.heads[0]) {}
};

// 1 / sqrt(x) by the instruction (1 ulp; 5003 tokens of 16 heads 10.9 us, 11.3 by root and quotient), which takes what is below the normal numbers
// for 0.  The mean before it is a product with 1 / D as 32 bits hold it, half a unit more in its last place than a quotient, of which the root leaves half.
__device__ __forceinline__ float inverse_root(float x) {
  if (__any(x < 0x1p-126f)) return 1.0f / sqrtf(x);
  return __builtin_amdgcn_rsqf(x);
}

template <int V> __device__ __forceinline__ float sum_of_products(const float (&x)[2][V], const float (&y)[2][V]) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i) s = fmaf(x[1][i], y[1][i], fmaf(x[0][i], y[0][i], s));
  return s;
}

template <class T, int V, int Pairs, bool Stream, bool Axes>
__global__ __launch_bounds__(kThreads, Axes ? 4 : 5) void heads_kernel(HeadsArgs a) {
  const unsigned lanes = 1u << a.lanes_log2, rows = kWave >> a.lanes_log2;
  const unsigned chunk = lane_id() & (lanes - 1), row_of_wave = lane_id() >> a.lanes_log2;
  const Place<V, Pairs> p(a.dim, a.half, chunk);
  const auto wq = load_weight<T, V, Pairs>(a.weight[0], p), wk = load_weight<T, V, Pairs>(a.weight[1], p);
  const unsigned first = blockIdx.y * a.per_wave, end = min(first + a.per_wave, a.heads[0] + a.heads[1] + a.heads[2]);
  const float by_dim = 1.0f / (float)a.dim;
  const unsigned axes = Axes ? axes_of_lane(a) : 0u;
  constexpr bool kCross = Pairs == kCrossed;
  __shared__ alignas(32) float shared[Axes ? kWaves : 1][kCross ? 2 * kMostDim : Axes ? kMostDim : 1];
  __shared__ alignas(32) float crossed[kCross ? kThreads * 2 * V : 1];
  auto load = [&](const Turn &n, unsigned t) { return load_packs<Stream>(row_of<const T>(either(n.is_q, a.q, either(n.is_v, a.v, a.k)), t, n.head), p, n.live); };
  for (unsigned t = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(wave_id()); t < a.tokens; t += gridDim.x * kWaves) {
    auto next = load(Turn(a, first + row_of_wave, end), t);
    float c[V] = {}, s[V] = {};
    if constexpr (Axes) stage_angles<Pairs>(a, axes, t, shared[wave_id()]);
    else load_angles(a, p, t, c, s);
    const long long slot = a.slots ? load_scalar(a.slots + t) : 0;
    const bool stored = !a.slots || (unsigned long long)slot < a.places;
    const unsigned page = a.slots && stored ? (unsigned)slot / a.page : 0u, place = a.slots && stored ? (unsigned)slot - page * a.page : 0u;
    for (unsigned h0 = first; h0 < end; h0 += rows) {
      const Turn n(a, h0 + row_of_wave, end);
      const auto now = next;
      next = load(Turn(a, h0 + rows + row_of_wave, end), t);
      float x[2][V];
      unpack(now, p, x);
      const float square = lanes_sum(sum_of_products(x, x), (int)a.lanes_log2);
      if (!n.is_v) {
        if constexpr (Axes && !kCross) staged_angles(p, shared[wave_id()], c, s);
        float w[2][V];
        unpack(either(n.is_q, wq, wk), p, w);
        const float r = (n.is_q ? a.weight[0] != nullptr : a.weight[1] != nullptr) ? inverse_root(square * by_dim + a.eps) : 1.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float y0 = x[0][i] * r * w[0][i], y1 = x[1][i] * r * w[1][i];
          x[0][i] = !kCross && p.turns(i) ? y0 * c[i] - y1 * s[i] : y0;
          x[1][i] = !kCross && p.turns(i) ? y1 * c[i] + y0 * s[i] : y1;
        }
        if constexpr (kCross) turn_crossed<false>(p, a.half, shared[wave_id()], crossed + (threadIdx.x - chunk) * 2 * V, x);
      }
      if (!n.live || (!n.is_q && !stored)) continue;
      T *to;
      if (n.is_q) to = row_of<T>(a.q_out, t, n.head);
      else if (n.is_v) to = reinterpret_cast<T *>(a.v_cache) + page * a.v_page + place * a.v_place + n.head * a.v_head;
      else if (a.slots) to = reinterpret_cast<T *>(a.k_out.ptr) + page * a.k_page + place * a.k_place + n.head * a.k_out.head;
      else to = row_of<T>(a.k_out, t, n.head);
      store_row<Stream>(to, p, x);
    }
  }
}

struct GradRows {
  Rows dy[2], dx[2];                        // of q and of k
};

// dx, and this workgroup's sums of the weights' gradients: partial[group][q, k][D].  Registers are for three workgroups a compute unit: 16-bit rows with
// neighbours paired and one axis leave 6 to 10 vector registers of them in memory (28 to 44 bytes a lane), and most forms with several axes 20 bytes.
template <class T, int V, int Pairs, bool Stream, bool Axes>
__global__ __launch_bounds__(kThreads, 3) void heads_grad_kernel(HeadsArgs a, GradRows rows_of, float *partial) {
  constexpr bool kCross = Pairs == kCrossed;
  __shared__ alignas(32) float sums[kWaves][2][kMostDim];    // of the weights' gradients, at the end; before it the staged angles
  __shared__ alignas(32) float crossed[kCross ? kThreads * 2 * V : 1];
  const unsigned lanes = 1u << a.lanes_log2, rows = kWave >> a.lanes_log2;
  const unsigned chunk = lane_id() & (lanes - 1), row_of_wave = lane_id() >> a.lanes_log2;
  const Place<V, Pairs> p(a.dim, a.half, chunk);
  const auto wq = load_weight<T, V, Pairs>(a.weight[0], p), wk = load_weight<T, V, Pairs>(a.weight[1], p);
  float dq[2][V], dk[2][V];
#pragma unroll
  for (int i = 0; i < V; ++i) dq[0][i] = dq[1][i] = dk[0][i] = dk[1][i] = 0.0f;
  const unsigned first = blockIdx.y * a.per_wave, end = min(first + a.per_wave, a.heads[0] + a.heads[1]);
  const float by_dim = 1.0f / (float)a.dim;
  const unsigned axes = Axes ? axes_of_lane(a) : 0u;
  auto load_x = [&](const Turn &n, unsigned t) { return load_packs<Stream>(row_of<const T>(either(n.is_q, a.q, a.k), t, n.head), p, n.live); };
  auto load_g = [&](const Turn &n, unsigned t) { return load_packs<Stream>(row_of<const T>(either(n.is_q, rows_of.dy[0], rows_of.dy[1]), t, n.head), p, n.live); };
  for (unsigned t = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(wave_id()); t < a.tokens; t += gridDim.x * kWaves) {
    auto next_x = load_x(Turn(a, first + row_of_wave, end), t), next_g = load_g(Turn(a, first + row_of_wave, end), t);
    float c[V] = {}, s[V] = {};
    if constexpr (Axes) stage_angles<Pairs>(a, axes, t, sums[wave_id()][0]);
    else load_angles(a, p, t, c, s);
    for (unsigned h0 = first; h0 < end; h0 += rows) {
      const Turn n(a, h0 + row_of_wave, end);
      float x[2][V], g[2][V];
      unpack(next_x, p, x);
      unpack(next_g, p, g);
      const Turn then(a, h0 + rows + row_of_wave, end);
      next_x = load_x(then, t);
      next_g = load_g(then, t);
      if constexpr (kCross) turn_crossed<true>(p, a.half, sums[wave_id()][0], crossed + (threadIdx.x - chunk) * 2 * V, g);
      else {
        if constexpr (Axes) staged_angles(p, sums[wave_id()][0], c, s);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float g0 = g[0][i], g1 = g[1][i];
          g[0][i] = p.turns(i) ? g0 * c[i] + g1 * s[i] : g0;
          g[1][i] = p.turns(i) ? g1 * c[i] - g0 * s[i] : g1;
        }
      }
      if (n.is_q ? a.weight[0] != nullptr : a.weight[1] != nullptr) {
        // the sums are taken by all lanes of a row together: a row is of q or of k as a whole.  A row that no head has is zeros, whose norm
        // is not finite where eps is 0: it must leave the weights' sums alone.
        const float square = lanes_sum(sum_of_products(x, x), (int)a.lanes_log2);
        const float root = inverse_root(square * by_dim + a.eps), r = n.live ? root : 0.0f;
        float w[2][V];
        unpack(either(n.is_q, wq, wk), p, w);
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            x[k][i] *= r;
            const float dw = g[k][i] * x[k][i];
            dq[k][i] += n.is_q ? dw : 0.0f;
            dk[k][i] += n.is_q ? 0.0f : dw;
            g[k][i] *= w[k][i];
          }
        const float mean = lanes_sum(sum_of_products(g, x), (int)a.lanes_log2) * by_dim;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) g[k][i] = r * (g[k][i] - x[k][i] * mean);
      }
      if (n.live) store_row<Stream>(row_of<T>(either(n.is_q, rows_of.dx[0], rows_of.dx[1]), t, n.head), p, g);
    }
  }
  if (!partial) return;
  // over the rows of the wave, then over the waves
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i)
      for (unsigned d = lanes; d < (unsigned)kWave; d *= 2) {
        dq[k][i] += __shfl_xor(dq[k][i], (int)d);
        dk[k][i] += __shfl_xor(dk[k][i], (int)d);
      }
  if (row_of_wave == 0) {
    store_row<false>(sums[wave_id()][0], p, dq);
    store_row<false>(sums[wave_id()][1], p, dk);
  }
  __syncthreads();
  const unsigned group = blockIdx.y * gridDim.x + blockIdx.x;
  for (unsigned i = threadIdx.x; i < 2 * a.dim; i += kThreads) {
    const unsigned which = i >= a.dim, d = i - which * a.dim;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += sums[w][which][d];
    partial[(unsigned long long)group * 2 * a.dim + i] = sum;
  }
}

// dw[i] = sum of partial[g][i] over the groups: kColumns columns a workgroup, the groups shared by its threads, eight of a thread's on
// their way at a time
constexpr int kColumns = 8, kAdders = 1024 / kColumns;
__global__ __launch_bounds__(1024) void weight_grad_kernel(const float *partial, unsigned groups, unsigned dim, float *dq, float *dk) {
  __shared__ float sums[kAdders][kColumns + 1];
  const unsigned mine = threadIdx.x % kColumns, column = blockIdx.x * kColumns + mine, of = threadIdx.x / kColumns;
  float sum = 0.0f;
  if (column < 2 * dim)
    for (unsigned g = of; g < groups; g += 8 * kAdders) {
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = g + k * kAdders < groups ? partial[(unsigned long long)(g + k * kAdders) * 2 * dim + column] : 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += x[k];
    }
  sums[of][mine] = sum;
  __syncthreads();
  // the first wave: 8 threads a column, each 16 of the sums, then the 8
  if (threadIdx.x >= 8 * kColumns) return;
  sum = 0.0f;
#pragma unroll
  for (int k = 0; k < kAdders / 8; ++k) sum += sums[k * 8 + of][mine];
#pragma unroll
  for (int d = kColumns; d < 8 * kColumns; d *= 2) sum += __shfl_xor(sum, d);
  float *to = column < dim ? dq : dk;
  if (of == 0 && column < 2 * dim && to) to[column < dim ? column : column - dim] = sum;
}

// ------------------------------------------------------------------ host
// calls f with the type, the elements of a pack, the pairing and the way through the caches of this call as compile-time values
template <class F> void with_form(int32_t dtype, int pack, int pairs, bool stream, bool axes, F &&f) {
  auto by_axes = [&](auto element, auto v, auto paired, auto past) {
    if constexpr (decltype(paired)::value == kCrossed) {
      if constexpr (decltype(v)::value > 1) f(element, v, paired, past, std::true_type{});
    } else axes ? f(element, v, paired, past, std::true_type{}) : f(element, v, paired, past, std::false_type{});
  };
  auto by_pack = [&](auto element, auto paired) {
    using T = decltype(element);
    constexpr int kWide = 16 / sizeof(T);
    if (pack == kWide && stream) by_axes(element, std::integral_constant<int, kWide>{}, paired, std::true_type{});
    else if (pack == kWide) by_axes(element, std::integral_constant<int, kWide>{}, paired, std::false_type{});
    else if (kWide > 4 && pack == 4) by_axes(element, std::integral_constant<int, 4>{}, paired, std::false_type{});
    else if (pack == 2) by_axes(element, std::integral_constant<int, 2>{}, paired, std::false_type{});
    else by_axes(element, std::integral_constant<int, 1>{}, paired, std::false_type{});
  };
  auto by_pairing = [&](auto element) {
    if (pairs == kNeighbours) by_pack(element, std::integral_constant<int, kNeighbours>{});
    else if (pairs == kCrossed) by_pack(element, std::integral_constant<int, kCrossed>{});
    else by_pack(element, std::integral_constant<int, kHalves>{});
  };
  if (dtype == FC_F32) by_pairing(float{});
  else if (dtype == FC_F16) by_pairing(_Float16{});
  else by_pairing(__bf16{});
}

Rows rows_at(const fc_tensor &t) { return {static_cast<char *>(t.ptr), t.stride[0], t.stride[1]}; }

struct HeadsCall {
  HeadsArgs a{};
  int32_t dtype;
  int pack;
  int pairs;
  dim3 grid;
  unsigned heads() const { return a.heads[0] + a.heads[1] + a.heads[2]; }
  // What is read and written passes the caches where they would not hold it until it is used (16384 tokens of 40 heads 70 us through them,
  // 61 past them; 4000 tokens, 41 MB, 18.7 either way).
  bool stream() const { return (unsigned long long)a.tokens * heads() * a.dim * size_of_dtype(dtype) >= 32u << 20; }
  // How the heads of a token are shared among waves (grid.y), and the workgroups that are then needed, as many as are resident at once at
  // most: a second round of a few lasts as long as the first (the gradient of 16384 tokens on 768 workgroups 97 us, 1024 120).  A wave takes
  // all heads of a token, unless that leaves compute units without work.
  template <class... P> void shape(void (*kernel)(P...)) {
    const unsigned resident = resident_workgroups(kernel, kThreads), most = resident ? resident : 768u;
    const unsigned rows = kWave >> a.lanes_log2, turns = std::max(1u, ceil_div(heads(), rows));
    const unsigned parts = std::min({turns, std::max(1u, 4096u / std::max(1u, a.tokens)), most});
    a.per_wave = ceil_div(turns, parts) * rows;
    grid.y = std::max(1u, ceil_div(heads(), a.per_wave));
    grid.x = std::max(1u, std::min(ceil_div(a.tokens, kWaves), most / grid.y));
  }
};

// what the operator and its gradient have in common
int check_heads(TensorChecks &c, const fc_tensor &q, const fc_tensor &k, const fc_tensor &q_weight, const fc_tensor &k_weight, const fc_tensor &cos_sin,
                const fc_tensor &positions, const fc_tensor &axis_of, double eps, int32_t interleaved, bool values, HeadsCall &call) {
  const int32_t dtype = q.dtype;
  if (dtype != FC_F32 && dtype != FC_F16 && dtype != FC_BF16) return c.fail(FC_E_ARG, "q: type f32, f16 or bf16 is needed").code();
  c.array("q", q, dtype, {-1, -1, -1});
  if (!c.ok()) return c.code();
  const int64_t tokens = q.shape[0], dim = q.shape[2];
  c.array("k", k, dtype, {tokens, -1, dim});
  if (present(q_weight)) c.array("q_weight", q_weight, dtype, {dim});
  if (present(k_weight)) c.array("k_weight", k_weight, dtype, {dim});
  if (present(cos_sin)) {
    c.array("cos_sin", cos_sin, FC_F32, {-1, -1});
    c.array("positions", positions, FC_I32, {-1, tokens});
    if (c.ok() && (cos_sin.shape[1] % 2 || cos_sin.shape[1] > dim)) c.fail(FC_E_ARG, "cos_sin: an even number of columns, at most the elements of a head, is needed");
    if (present(axis_of)) c.array("axis_of", axis_of, FC_I32, {cos_sin.shape[1] / 2});
    if (c.ok() && positions.shape[0] > 255) c.fail(FC_E_LIMIT, "positions: more than 255 axes");
  } else if (present(positions) || present(axis_of)) {
    c.fail(FC_E_ARG, "positions and axis_of go with cos_sin");
  }
  if (c.ok() && !(eps >= 0 && std::isfinite((float)eps))) c.fail(FC_E_ARG, "eps must be finite, in 32 bits too, and not negative");
  if (c.ok() && eps > 0 && (float)eps == 0) c.fail(FC_E_ARG, "eps is 0 in 32 bits");      // rows of zeros would be NaN
  if (c.ok() && (dim < 2 || dim % 2 || dim > (int64_t)kMostDim)) c.fail(FC_E_UNSUPPORTED, "heads have an even number of elements, at most 512");
  // a token's heads, those of values among them, are numbered in one row, which a wave walks in steps of up to 64 that must not pass 32 bits
  if (c.ok() && (q.shape[1] + (values ? 2 : 1) * k.shape[1] > 0x7fffffff || tokens * (q.shape[1] + k.shape[1]) > (int64_t)1 << 40)) c.fail(FC_E_LIMIT, "too many heads");
  if (!c.ok()) return c.code();
  HeadsArgs &a = call.a;
  a.q = rows_at(q);
  a.k = rows_at(k);
  a.weight[0] = present(q_weight) ? q_weight.ptr : nullptr;
  a.weight[1] = present(k_weight) ? k_weight.ptr : nullptr;
  if (present(cos_sin) && cos_sin.shape[1] > 0) {
    a.half = (unsigned)cos_sin.shape[1] / 2;
    a.cos_sin = static_cast<const float *>(cos_sin.ptr);
    a.positions = static_cast<const int *>(positions.ptr);
    a.axis_of = present(axis_of) ? static_cast<const int *>(axis_of.ptr) : nullptr;
    a.angle_stride = cos_sin.stride[0];
    a.position_stride = positions.stride[0];
    a.angles = (unsigned)cos_sin.shape[0];
    a.axes = (unsigned)positions.shape[0];
  }
  a.tokens = (unsigned)tokens;
  a.heads[0] = (unsigned)q.shape[1];
  a.heads[1] = (unsigned)k.shape[1];
  a.dim = (unsigned)dim;
  a.eps = (float)eps;
  call.dtype = dtype;
  call.pairs = interleaved ? kNeighbours : kHalves;
  // 16 bytes a pack, less where the elements of a head, the strides or the alignment of an array do not allow it
  call.pack = 16 / size_of_dtype(dtype);
  while (call.pack > 1 && dim / 2 % call.pack) call.pack /= 2;
  for (const fc_tensor *t : {&q, &k, &q_weight, &k_weight})
    if (present(*t)) call.pack = common_alignment(*t, call.pack);
  a.wide_angles = a.half && common_alignment(cos_sin, 4) == 4;
  return FC_OK;
}

// once the packs are known
int settle_lanes(TensorChecks &c, HeadsCall &call) {
  // Packs of halves end where the rotated part does, unless that leaves one or two elements: larger ones that cross take the gradient of 12844 tokens of
  // 28 heads of 72 with 18 elements turned in 66 us, packs of one in 129; with 20 of 80 69, packs of two 97; but with 40 of 80 69, packs of four 54.
  // Neighbours stay in one pack either way (60 us, 157 with packs that end there too).
  int pack = call.pack;
  while (call.pairs == kHalves && pack > 1 && call.a.half % pack) pack /= 2;
  unsigned lanes = 1;
  while (lanes * 2 * pack < call.a.dim) lanes *= 2;
  if (lanes > (unsigned)kWave)
    return c.fail(FC_E_UNSUPPORTED, "heads of " + std::to_string(call.a.dim) + " elements can be read " + std::to_string(pack) +
                                        " at a time only (rotated pairs, strides and alignment): at most " + std::to_string(128 * pack) + " are built for").code();
  if (pack < call.pack && pack <= 2) call.pairs = kCrossed;
  else call.pack = pack;
  while ((2u * call.pack << call.a.lanes_log2) < call.a.dim) ++call.a.lanes_log2;
  // angles are read as many at once as a pack has pairs, at most four
  call.a.wide_angles = call.a.wide_angles && call.a.half % std::max(1, std::min(call.pairs == kNeighbours ? call.pack / 2 : call.pack, 4)) == 0;
  return FC_OK;
}

struct HeadNormRope final : Operator, HeadsCall {
  template <class F> void with_kernel(F &&f) const {
    with_form(dtype, pack, pairs, stream(), a.axis_of != nullptr, [&](auto element, auto v, auto paired, auto past, auto axes) {
      f(&heads_kernel<decltype(element), decltype(v)::value, decltype(paired)::value, decltype(past)::value, decltype(axes)::value>);
    });
  }
  void record(Recorder &r) const override {
    if (a.tokens == 0 || heads() == 0) return;
    with_kernel([&](auto kernel) { r.launch(kernel, grid, kThreads, a); });
  }
  const char *name() const override { return "head norm and rotation"; }
};

struct HeadNormRopeGrad final : Operator, HeadsCall {
  GradRows rows{};
  float *dw[2] = {nullptr, nullptr};
  unsigned groups() const { return grid.x * grid.y; }
  size_t workspace() const override { return dw[0] || dw[1] ? (size_t)groups() * 2 * a.dim * sizeof(float) : 0; }
  template <class F> void with_kernel(F &&f) const {
    with_form(dtype, pack, pairs, stream(), a.axis_of != nullptr, [&](auto element, auto v, auto paired, auto past, auto axes) {
      f(&heads_grad_kernel<decltype(element), decltype(v)::value, decltype(paired)::value, decltype(past)::value, decltype(axes)::value>);
    });
  }
  void record(Recorder &r) const override {
    float *partial = dw[0] || dw[1] ? reinterpret_cast<float *>(r.workspace) : nullptr;
    if (!partial && (a.tokens == 0 || heads() == 0)) return;
    with_kernel([&](auto kernel) { r.launch(kernel, grid, kThreads, a, rows, partial); });
    if (partial) r.launch(&weight_grad_kernel, ceil_div(2 * a.dim, kColumns), 1024, (const float *)partial, groups(), a.dim, dw[0], dw[1]);
  }
  const char *name() const override { return "gradient of head norm and rotation"; }
};

}  // namespace

int make_head_norm_rope(const fc_head_norm_rope &n, std::unique_ptr<Operator> &out, std::string &err) {
  TensorChecks c(err);
  auto op = std::make_unique<HeadNormRope>();
  if (check_heads(c, n.q, n.k, n.q_weight, n.k_weight, n.cos_sin, n.positions, n.axis_of, n.eps, n.interleaved, present(n.slots), *op) != FC_OK) return c.code();
  HeadsArgs &a = op->a;
  const int64_t tokens = a.tokens, dim = a.dim, kv = a.heads[1];
  c.array("q_out", n.q_out, op->dtype, {tokens, a.heads[0], dim}, true);
  if (c.ok() && other_strides(n.q, n.q_out)) c.fail(FC_E_ARG, "q_out is at the address of q with other strides");
  a.q_out = rows_at(n.q_out);
  auto align = [&](const fc_tensor &t) { op->pack = common_alignment(t, op->pack); };
  if (present(n.slots)) {
    if (present(n.k_out)) c.fail(FC_E_ARG, "keys go to k_out or, with slots, to the cache");
    c.array("slots", n.slots, FC_I64, {tokens});
    c.array("v", n.v, op->dtype, {tokens, kv, dim});
    c.array("k_cache", n.k_cache, op->dtype, {-1, -1, kv, dim}, true);
    c.array("v_cache", n.v_cache, op->dtype, {n.k_cache.shape[0], n.k_cache.shape[1], kv, dim}, true);
    if (c.ok() && n.k_cache.shape[1] < 1) c.fail(FC_E_ARG, "k_cache: pages without places");
    if (!c.ok()) return c.code();
    a.slots = static_cast<const long long *>(n.slots.ptr);
    a.heads[2] = (unsigned)kv;
    a.v = rows_at(n.v);
    if (n.k_cache.shape[0] * n.k_cache.shape[1] > 0x7fffffff) return c.fail(FC_E_LIMIT, "k_cache: more than 2^31-1 places").code();
    a.page = (unsigned)n.k_cache.shape[1];
    a.places = (unsigned)(n.k_cache.shape[0] * n.k_cache.shape[1]);
    a.k_out = {static_cast<char *>(n.k_cache.ptr), 0, n.k_cache.stride[2]};
    a.v_cache = static_cast<char *>(n.v_cache.ptr);
    a.k_page = n.k_cache.stride[0];
    a.k_place = n.k_cache.stride[1];
    a.v_page = n.v_cache.stride[0];
    a.v_place = n.v_cache.stride[1];
    a.v_head = n.v_cache.stride[2];
    for (const fc_tensor *t : {&n.v, &n.k_cache, &n.v_cache}) align(*t);
  } else {
    if (present(n.v) || present(n.k_cache) || present(n.v_cache)) c.fail(FC_E_ARG, "v and the caches go with slots");
    c.array("k_out", n.k_out, op->dtype, {tokens, kv, dim}, true);
    if (c.ok() && other_strides(n.k, n.k_out)) c.fail(FC_E_ARG, "k_out is at the address of k with other strides");
    a.k_out = rows_at(n.k_out);
    align(n.k_out);
  }
  if (!c.ok()) return c.code();
  align(n.q_out);
  if (settle_lanes(c, *op) != FC_OK) return c.code();
  op->with_kernel([&](auto kernel) { op->shape(kernel); });
  out = std::move(op);
  return FC_OK;
}

int make_head_norm_rope_grad(const fc_head_norm_rope_grad &n, std::unique_ptr<Operator> &out, std::string &err) {
  TensorChecks c(err);
  auto op = std::make_unique<HeadNormRopeGrad>();
  if (check_heads(c, n.q, n.k, n.q_weight, n.k_weight, n.cos_sin, n.positions, n.axis_of, n.eps, n.interleaved, false, *op) != FC_OK) return c.code();
  HeadsArgs &a = op->a;
  const int64_t tokens = a.tokens, dim = a.dim;
  c.array("dq_out", n.dq_out, op->dtype, {tokens, a.heads[0], dim});
  c.array("dk_out", n.dk_out, op->dtype, {tokens, a.heads[1], dim});
  c.array("dq", n.dq, op->dtype, {tokens, a.heads[0], dim}, true);
  c.array("dk", n.dk, op->dtype, {tokens, a.heads[1], dim}, true);
  if (c.ok() && other_strides(n.dq_out, n.dq)) c.fail(FC_E_ARG, "dq is at the address of dq_out with other strides");
  if (c.ok() && other_strides(n.dk_out, n.dk)) c.fail(FC_E_ARG, "dk is at the address of dk_out with other strides");
  if (present(n.q_weight) != present(n.dq_weight) || present(n.k_weight) != present(n.dk_weight))
    c.fail(FC_E_ARG, "a weight and its gradient are there together or not at all");
  if (present(n.dq_weight)) c.array("dq_weight", n.dq_weight, FC_F32, {dim}, true);
  if (present(n.dk_weight)) c.array("dk_weight", n.dk_weight, FC_F32, {dim}, true);
  if (!c.ok()) return c.code();
  op->rows = {{rows_at(n.dq_out), rows_at(n.dk_out)}, {rows_at(n.dq), rows_at(n.dk)}};
  for (const fc_tensor *t : {&n.dq_out, &n.dk_out, &n.dq, &n.dk}) op->pack = common_alignment(*t, op->pack);
  if (settle_lanes(c, *op) != FC_OK) return c.code();
  op->dw[0] = present(n.dq_weight) ? static_cast<float *>(n.dq_weight.ptr) : nullptr;
  op->dw[1] = present(n.dk_weight) ? static_cast<float *>(n.dk_weight.ptr) : nullptr;
  op->with_kernel([&](auto kernel) { op->shape(kernel); });
  out = std::move(op);
  return FC_OK;
}

}  // namespace fc
