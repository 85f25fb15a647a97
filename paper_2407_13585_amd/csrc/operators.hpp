// Operators of a serving cache (include/fc.h, fc_operator): what their translation units share.  Host side: checks of the
// caller's arrays and the launches an operator consists of; device side: element types and the steps across a few lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <memory>
#include <string>
#include <tuple>
#include <utility>
#include <vector>

#include "../../include/fc.h"
#include "prim.hpp"
#include "registry.hpp"

namespace fc {

// ------------------------------------------------------------------ host
// Where an operator's launches go, and the memory they share.
struct Recorder {
  std::vector<RecordedLaunch> &launches;
  char *workspace;                 // DEVICE: what workspace() asked for
  unsigned *counters;              // DEVICE: kCounters of them, 0 between launches
  const char *what;                // the operator, for the message of a launch that fails

  template <class... P, class... A> void launch(void (*kernel)(P...), dim3 grid, unsigned threads, const A &...a) {
    keep(kernel, grid, dim3(threads), std::make_shared<std::tuple<P...>>(a...), std::index_sequence_for<P...>());
  }

 private:
  template <class... P, size_t... I>
  void keep(void (*kernel)(P...), dim3 grid, dim3 block, std::shared_ptr<std::tuple<P...>> values, std::index_sequence<I...>) {
    RecordedLaunch r;
    r.kernel = reinterpret_cast<const void *>(kernel);
    r.grid = grid;
    r.block = block;
    r.args = {static_cast<void *>(&std::get<I>(*values))...};
    r.values = std::move(values);
    r.what = what;
    launches.push_back(std::move(r));
  }
};

// A checked operator.
struct Operator {
  virtual ~Operator() = default;
  virtual size_t workspace() const { return 0; }        // bytes of scratch behind the control block
  virtual void record(Recorder &r) const = 0;           // the launches, none where there is nothing to do
  virtual const char *name() const = 0;
};
using OperatorList = std::vector<std::unique_ptr<Operator>>;

int make_page_map(const fc_page_map &a, std::unique_ptr<Operator> &out, std::string &err);
int make_head_norm_rope(const fc_head_norm_rope &a, std::unique_ptr<Operator> &out, std::string &err);
int make_head_norm_rope_grad(const fc_head_norm_rope_grad &a, std::unique_ptr<Operator> &out, std::string &err);
int make_paged_attention(const fc_paged_attention &a, std::unique_ptr<Operator> &out, std::string &err);

int check_operators(const fc_operator *ops, int32_t n, OperatorList &out, std::string &err);
size_t operators_scratch_bytes(const OperatorList &list);
int record_operators(const OperatorList &list, void *scratch, size_t scratch_bytes, std::vector<RecordedLaunch> &out, std::string &err);

// One array of a call against what the operator needs of it.  The first that is wrong is reported.
class TensorChecks {
 public:
  explicit TensorChecks(std::string &err) : err_(err) {}
  // shape: -1 = any extent.  written: elements must lie apart.
  TensorChecks &array(const char *name, const fc_tensor &t, int32_t dtype, std::initializer_list<int64_t> shape, bool written = false);
  TensorChecks &fail(int code, const std::string &message);
  bool ok() const { return code_ == FC_OK; }
  int code() const { return code_; }

 private:
  std::string &err_;
  int code_ = FC_OK;
};

inline bool present(const fc_tensor &t) { return t.rank != 0; }
// Whether `out`, of the shape of `in` and at its address, lies otherwise than `in`, so that rows would be written over before they are
// read.  An axis along which `in` is one row for all is left to the caller.
inline bool other_strides(const fc_tensor &in, const fc_tensor &out) {
  bool differ = false, empty = false;
  for (int k = 0; k < in.rank; ++k) {
    differ |= in.shape[k] > 1 && in.stride[k] != 0 && in.stride[k] != out.stride[k];
    empty |= in.shape[k] == 0;
  }
  return in.ptr == out.ptr && differ && !empty;
}
inline int size_of_dtype(int32_t dtype) { return dtype == FC_I64 ? 8 : dtype == FC_F16 || dtype == FC_BF16 ? 2 : 4; }
// the largest power of two, `most` at most, that the base and all strides but the innermost (in elements) are multiples of
int common_alignment(const fc_tensor &t, int most);

inline unsigned ceil_div(unsigned long long a, unsigned long long b) { return (unsigned)((a + b - 1) / b); }

// ------------------------------------------------------------------ device
template <class T, int N> using Vec = T __attribute__((ext_vector_type(N)));      // aligned to its size

// Stream: past the caches, for what is used once (16 bytes)
template <class T, int N, bool Stream = false> __device__ __forceinline__ Vec<T, N> load_vec(const T *p) {
  if constexpr (Stream) return __builtin_bit_cast(Vec<T, N>, __builtin_nontemporal_load(reinterpret_cast<const Vec<unsigned, 4> *>(p)));
  else return *reinterpret_cast<const Vec<T, N> *>(p);
}
template <class T, int N, bool Stream = false> __device__ __forceinline__ void store_vec(T *p, Vec<T, N> v) {
  if constexpr (Stream) __builtin_nontemporal_store(__builtin_bit_cast(Vec<unsigned, 4>, v), reinterpret_cast<Vec<unsigned, 4> *>(p));
  else *reinterpret_cast<Vec<T, N> *>(p) = v;
}

// an element that this kernel does not write, for the whole wave: through the scalar unit, which has a counter of its own to wait for
template <class T> __device__ __forceinline__ T load_scalar(const T *p) {
  return *reinterpret_cast<const T __attribute__((address_space(4))) *>(reinterpret_cast<uintptr_t>(p));
}

// Sum over groups of 2^log2 neighbouring lanes, every lane gets it.  Up to 16 lanes by DPP: after the steps within four lanes, the
// mirror of eight and of sixteen bring the other half's sum.
__device__ __forceinline__ float lanes_sum(float v, int log2) {
  if (log2 >= 1) v += dpp_move<0xb1>(0.0f, v);         // quad_perm 1,0,3,2
  if (log2 >= 2) v += dpp_move<0x4e>(0.0f, v);         // quad_perm 2,3,0,1
  if (log2 >= 3) v += dpp_move<0x141>(0.0f, v);        // row_half_mirror
  if (log2 >= 4) v += dpp_move<0x140>(0.0f, v);        // row_mirror
  if (log2 >= 5) v += __shfl_xor(v, 16);
  if (log2 >= 6) v += __shfl_xor(v, 32);
  return v;
}

}  // namespace fc
