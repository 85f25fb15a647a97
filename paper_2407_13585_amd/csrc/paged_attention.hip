// Attention over one table a request (include/fc.h, fc_paged_attention), and what all forms of attention check and launch.
#include "attention.hpp"

#include <algorithm>
#include <cmath>

namespace fc {

template AttentionKernel attention_kernel_of<Form::kPlain>(int32_t, unsigned, bool);
extern template AttentionKernel attention_kernel_of<Form::kHeads>(int32_t, unsigned, bool);
extern template AttentionKernel attention_kernel_of<Form::kAfterPrefix>(int32_t, unsigned, bool);

AttentionKernel Attention::kernel() const {
  if (form == Form::kHeads) return attention_kernel_of<Form::kHeads>(dtype, a.dim, even);
  if (form == Form::kAfterPrefix) return attention_kernel_of<Form::kAfterPrefix>(dtype, a.dim, even);
  return attention_kernel_of<Form::kPlain>(dtype, a.dim, even);
}

void Attention::settle_workers() {
  const unsigned resident = resident_workgroups(kernel(), kThreads);
  a.workers = std::max(1u, std::min({resident ? resident : 512u, kCounters / 2u, most_units}));
  // a wave's step reads 128 D bytes: 16 kB under way for each of four waves are enough
  const int units = device_compute_units();
  a.streams = even ? std::min(a.workers, (units > 0 ? (unsigned)units : 256u) * ceil_div(128, a.dim)) : a.workers;
}

size_t Attention::workspace() const { return 2 * (size_t)a.workers * piece_floats(a.group, a.dim) * sizeof(float); }

void Attention::record(Recorder &r) const {
  if (a.requests == 0 || a.group == 0) return;
  AttentionArgs args = a;
  args.pieces = reinterpret_cast<float *>(r.workspace);
  args.counters = r.counters;
  r.launch(kernel(), a.workers, kThreads, args);
}

int settle_attention(const fc_paged_attention &n, Attention &op, std::string &err) {
  TensorChecks c(err);
  const int32_t dtype = n.q.dtype;
  if (dtype != FC_F32 && dtype != FC_F16 && dtype != FC_BF16) return c.fail(FC_E_ARG, "q: type f32, f16 or bf16 is needed").code();
  c.array("q", n.q, dtype, {-1, -1, -1});
  const int64_t requests = n.q.shape[0], heads = n.q.shape[1], dim = n.q.shape[2];
  c.array("k_cache", n.k_cache, dtype, {-1, -1, -1, dim});
  const int64_t pages = n.k_cache.shape[0], page = n.k_cache.shape[1], kv = n.k_cache.shape[2];
  c.array("v_cache", n.v_cache, dtype, {pages, page, kv, dim});
  const bool by_head = op.form == Form::kHeads;
  if (by_head) {
    c.array("table", n.table, FC_I32, {requests, kv, -1});
    c.array("lengths", n.lengths, FC_I32, {requests, kv});
  } else {
    c.array("table", n.table, FC_I32, {requests, -1});
    c.array("lengths", n.lengths, FC_I32, {requests});
  }
  c.array("out", n.out, dtype, {requests, heads, dim}, true);
  if (present(n.lse)) c.array("lse", n.lse, FC_F32, {requests, heads}, true);
  if (!c.ok()) return c.code();
  if (page < 1) return c.fail(FC_E_ARG, "k_cache: pages without places").code();
  if (kv < 1 || heads % kv) return c.fail(FC_E_ARG, "the heads of q must be a multiple of those of the cache").code();
  if (dim < 8 || dim % 8 || dim > (int64_t)kMostDim) return c.fail(FC_E_UNSUPPORTED, "heads have a multiple of 8 elements, at most 256").code();
  if (!std::isfinite((float)n.scale)) return c.fail(FC_E_ARG, "scale must be finite, in 32 bits too").code();
  if (n.window < 0) return c.fail(FC_E_ARG, "window must not be negative").code();
  for (const fc_tensor *t : {&n.q, &n.k_cache, &n.v_cache})
    if (requests && pages && common_alignment(*t, 16 / size_of_dtype(dtype)) * size_of_dtype(dtype) != 16)
      return c.fail(FC_E_UNBOUND, "the rows of q and of the caches must be 16-byte aligned").code();
  // a workgroup counts the elements of a request without keys four at a time, and steps past the last
  if (heads * (dim / 4) > 0x7fffffff) return c.fail(FC_E_LIMIT, "a request's heads have more than 2^33 elements").code();
  // rows of lengths are counted in 31 bits
  if (by_head && requests * kv > 0x7fffffff) return c.fail(FC_E_LIMIT, "too many requests and key heads together").code();
  AttentionArgs &a = op.a;
  op.dtype = dtype;
  a.q = static_cast<const char *>(n.q.ptr);
  a.k = static_cast<const char *>(n.k_cache.ptr);
  a.v = static_cast<const char *>(n.v_cache.ptr);
  a.table = static_cast<const int *>(n.table.ptr);
  a.lengths = static_cast<const int *>(n.lengths.ptr);
  a.out = static_cast<char *>(n.out.ptr);
  a.lse = present(n.lse) ? static_cast<float *>(n.lse.ptr) : nullptr;
  a.q_request = n.q.stride[0];
  a.q_head = n.q.stride[1];
  a.out_request = n.out.stride[0];
  a.out_head = n.out.stride[1];
  a.lse_request = n.lse.stride[0];
  a.table_stride = n.table.stride[0];
  a.k_page = n.k_cache.stride[0];
  a.k_place = n.k_cache.stride[1];
  a.k_head = n.k_cache.stride[2];
  a.v_page = n.v_cache.stride[0];
  a.v_place = n.v_cache.stride[1];
  a.v_head = n.v_cache.stride[2];
  a.table_head = n.table.stride[1];
  a.length_request = n.lengths.stride[0];
  a.heads = (unsigned)kv;
  a.requests = (unsigned)(by_head ? requests * kv : requests);
  a.kv_heads = by_head ? 1u : (unsigned)kv;
  a.group = (unsigned)(heads / kv);
  a.tiles = ceil_div(a.group, kColumns);
  a.dim = (unsigned)dim;
  a.page = (unsigned)page;
  a.pages = (unsigned)pages;
  a.width = (unsigned)n.table.shape[by_head ? 2 : 1];
  a.window = (unsigned)n.window;
  // the places of a page apart and in order, so that a descriptor's end tells what is there
  op.even = page % 16 == 0 && std::min(a.k_place, a.v_place) >= dim && std::max(a.k_place, a.v_place) * 16 * size_of_dtype(dtype) < (int64_t)1 << 31;
  if (op.even) {
    // factor = ceil(2^(31 + s) / d), 2^s <= d: its error times n is below 2^(31 + s) for n below 2^30
    const unsigned d = a.page / 16, s = 31u - (unsigned)__builtin_clz(d);
    a.page_shift = 31 + s;
    a.page_factor = (unsigned)(((1ull << a.page_shift) + d - 1) / d);
  }
  a.scale = (float)n.scale;
  a.wide_out = common_alignment(n.out, 16 / size_of_dtype(dtype)) * size_of_dtype(dtype) == 16;
  // of a request, whose length is below 2^31 whatever its table could hold: one more where a window starts inside
  const uint64_t keys = std::min<uint64_t>((uint64_t)a.width * a.page, 0x7fffffffu);
  const unsigned units = ceil_div(keys, dtype == FC_F32 ? kUnit<float> : kUnit<_Float16>) + 1;
  unsigned most_units;
  if (__builtin_mul_overflow(units, a.requests, &most_units) || __builtin_mul_overflow(most_units, a.kv_heads, &most_units) ||
      __builtin_mul_overflow(most_units, a.tiles, &most_units) || most_units > 0x7fffffffu)
    return c.fail(FC_E_LIMIT, "too many requests, heads and pages of a request together").code();
  op.most_units = most_units;
  op.settle_workers();
  return FC_OK;
}

int make_paged_attention(const fc_paged_attention &n, std::unique_ptr<Operator> &out, std::string &err) {
  auto op = std::make_unique<Attention>();
  if (n.table.rank == 3) op->form = Form::kHeads;
  const int rc = settle_attention(n, *op, err);
  if (rc == FC_OK) out = std::move(op);
  return rc;
}

}  // namespace fc
