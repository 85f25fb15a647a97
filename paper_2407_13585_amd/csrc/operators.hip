// Operators of a serving cache: checks common to all of them, and lists of them in one scratch buffer.
#include "operators.hpp"

#include <algorithm>
#include <numeric>

namespace fc {

namespace {

const char *dtype_name(int32_t d) {
  switch (d) {
    case FC_F32: return "f32";
    case FC_I32: return "i32";
    case FC_F16: return "f16";
    case FC_BF16: return "bf16";
    case FC_I64: return "i64";
    default: return "unknown";
  }
}

// elements from the first to behind the last; apart: whether no two of them share memory (every stride is at least what the
// smaller ones span)
__int128 span_of(const fc_tensor &t, bool &apart) {
  int order[4] = {0, 1, 2, 3};
  std::sort(order, order + t.rank, [&](int a, int b) { return t.stride[a] < t.stride[b]; });
  __int128 span = 1;
  apart = true;
  for (int k = 0; k < t.rank; ++k) {
    const int d = order[k];
    if (t.shape[d] == 1) continue;
    if (t.stride[d] < span) apart = false;
    span += (__int128)t.stride[d] * (t.shape[d] - 1);
  }
  return span;
}

}  // namespace

TensorChecks &TensorChecks::fail(int code, const std::string &message) {
  if (ok()) { code_ = code; err_ = message; }
  return *this;
}

TensorChecks &TensorChecks::array(const char *name, const fc_tensor &t, int32_t dtype, std::initializer_list<int64_t> shape, bool written) {
  if (!ok()) return *this;
  const std::string who(name);
  if (t.rank < 0 || t.rank > 4) return fail(FC_E_ARG, who + ": rank out of range");
  if (t.rank != (int)shape.size()) return fail(FC_E_ARG, who + ": rank " + std::to_string(t.rank) + " where " + std::to_string(shape.size()) + " is needed");
  if (t.dtype != dtype) return fail(FC_E_ARG, who + ": type " + dtype_name(t.dtype) + " where " + dtype_name(dtype) + " is needed");
  bool empty = false;
  int k = 0;
  for (int64_t want : shape) {
    if (t.shape[k] < 0 || (want >= 0 && t.shape[k] != want))
      return fail(FC_E_ARG, who + ": extent " + std::to_string(k) + " is " + std::to_string(t.shape[k]) + (want >= 0 ? " where " + std::to_string(want) + " is needed" : ""));
    if (t.shape[k] > 0x7fffffff) return fail(FC_E_LIMIT, who + ": extent " + std::to_string(k) + " is above 2^31-1");
    if (t.shape[k] == 0) empty = true;
    if (t.shape[k] > 1 && t.stride[k] < 0) return fail(FC_E_ARG, who + ": stride " + std::to_string(k) + " is negative");
    ++k;
  }
  if (empty) return *this;
  if (t.shape[t.rank - 1] > 1 && t.stride[t.rank - 1] != 1) return fail(FC_E_ARG, who + ": the innermost stride must be 1");
  bool apart;
  if (span_of(t, apart) > (int64_t)1 << 44) return fail(FC_E_LIMIT, who + ": spans more than 2^44 elements");
  if (written && !apart) return fail(FC_E_ARG, who + ": is written, and its strides let elements share memory");
  if (!t.ptr) return fail(FC_E_UNBOUND, who + " has no memory");
  if ((uintptr_t)t.ptr % size_of_dtype(dtype)) return fail(FC_E_UNBOUND, who + " is not aligned to its elements");
  return *this;
}

int common_alignment(const fc_tensor &t, int most) {
  const int size = size_of_dtype(t.dtype);
  int a = most;
  auto allow = [&](uint64_t v) { while (a > 1 && v % a) a /= 2; };
  allow((uintptr_t)t.ptr / size);
  for (int k = 0; k + 1 < t.rank; ++k)
    if (t.shape[k] > 1) allow((uint64_t)t.stride[k]);
  return a;
}

int check_operators(const fc_operator *ops, int32_t n, OperatorList &out, std::string &err) {
  if (n < 0 || (n > 0 && !ops)) { err = "null list of operators"; return FC_E_ARG; }
  for (int i = 0; i < n; ++i) {
    std::unique_ptr<Operator> op;
    int rc = FC_OK;
    if (!ops[i].args) { err = "no arguments"; rc = FC_E_ARG; }
    else switch (ops[i].kind) {
      case FC_PAGE_MAP: rc = make_page_map(*static_cast<const fc_page_map *>(ops[i].args), op, err); break;
      case FC_HEAD_NORM_ROPE: rc = make_head_norm_rope(*static_cast<const fc_head_norm_rope *>(ops[i].args), op, err); break;
      case FC_HEAD_NORM_ROPE_GRAD: rc = make_head_norm_rope_grad(*static_cast<const fc_head_norm_rope_grad *>(ops[i].args), op, err); break;
      case FC_PAGED_ATTENTION: rc = make_paged_attention(*static_cast<const fc_paged_attention *>(ops[i].args), op, err); break;
      default: err = "unknown kind " + std::to_string(ops[i].kind); rc = FC_E_ARG;
    }
    if (rc != FC_OK) { err = "operator " + std::to_string(i) + ": " + err; return rc; }
    out.push_back(std::move(op));
  }
  return FC_OK;
}

size_t operators_scratch_bytes(const OperatorList &list) {
  size_t most = 0;                                  // the operators run one after the other: they share the workspace
  for (const auto &op : list) most = std::max(most, op->workspace());
  return FC_SCRATCH_CONTROL_BYTES + (most + 255) / 256 * 256;
}

int record_operators(const OperatorList &list, void *scratch, size_t scratch_bytes, std::vector<RecordedLaunch> &out, std::string &err) {
  if (!scratch || ((uintptr_t)scratch & 255u)) { err = "scratch must be a 256-byte aligned device buffer"; return FC_E_SCRATCH; }
  const size_t need = operators_scratch_bytes(list);
  if (scratch_bytes < need) { err = "scratch holds " + std::to_string(scratch_bytes) + " bytes where " + std::to_string(need) + " are needed"; return FC_E_SCRATCH; }
  for (const auto &op : list) {
    Recorder r{out, static_cast<char *>(scratch) + FC_SCRATCH_CONTROL_BYTES,
               reinterpret_cast<unsigned *>(static_cast<char *>(scratch) + kCountersOffset), op->name()};
    op->record(r);
  }
  return FC_OK;
}

}  // namespace fc
