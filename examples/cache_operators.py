"""A layer's attention as a server and as a trainer run it with the operators of the paged cache.

  Server: PageMap, HeadNormRope into the cache and PagedAttention, bound once and run step after step, requests coming and going.
  HeadNormRopeFunction: HeadNormRope and HeadNormRopeGrad as a differentiable function of PyTorch.

    python examples/cache_operators.py [--requests 64 --steps 64 --q-heads 32 --kv-heads 8 --dim 128 --page 16]

The layer is synthetic: random weights, and a step's output is the next step's input."""
import argparse
import os
import sys
import time

import torch
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_13585_amd as fc  # noqa: E402


def scratch_of(ops, device):
    return torch.zeros(fc.fc_operators_scratch_bytes(ops), dtype=torch.uint8, device=device)


def angle_table(positions, rotary, device, base=10000.0):
    turn = torch.arange(positions, device=device)[:, None] * base ** (-torch.arange(0, rotary, 2, device=device) / rotary)
    return torch.cat((turn.cos(), turn.sin()), dim=1).float()


class Server:
    """One layer's attention for `requests` requests of at most `max_len` tokens over a pool of `pages` pages."""

    def __init__(self, requests, max_len, pages, page=16, q_heads=32, kv_heads=8, dim=128, width=256, dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator(device).manual_seed(seed)
        i32 = dict(dtype=torch.int32, device=device)
        self.requests, self.page, self.q_heads, self.kv_heads, self.dim, self.dtype, self.device = requests, page, q_heads, kv_heads, dim, dtype, device
        # the layer
        self.qkv_weight = (torch.randn(width, (q_heads + 2 * kv_heads) * dim, generator=g, device=device) * width ** -0.5).to(dtype)
        self.out_weight = (torch.randn(q_heads * dim, width, generator=g, device=device) * (q_heads * dim) ** -0.5).to(dtype)
        self.q_norm = (1 + 0.1 * torch.randn(dim, generator=g, device=device)).to(dtype)
        self.k_norm = (1 + 0.1 * torch.randn(dim, generator=g, device=device)).to(dtype)
        self.angles = angle_table(max_len, dim, device)
        # the cache; lengths and cursor are there twice, before a step and after it
        self.k_cache = torch.zeros(pages, page, kv_heads, dim, dtype=dtype, device=device)
        self.v_cache = torch.zeros_like(self.k_cache)
        self.table = torch.full((requests, -(-max_len // page)), -1, **i32)
        self.pool = torch.arange(pages, **i32)
        self.lengths = [torch.zeros(requests, **i32) for _ in range(2)]
        self.cursor = [torch.tensor([0, pages], device=device) for _ in range(2)]
        self.unplaced = torch.zeros(1, dtype=torch.int64, device=device)
        self.now = 0
        # a decoding step, from each of the two states to the other
        self.hidden = torch.zeros(requests, width, dtype=dtype, device=device)
        self.one_each = torch.ones(requests, **i32)
        self.qkv = torch.empty(requests, self.qkv_weight.shape[1], dtype=dtype, device=device)
        self.heads_out = torch.empty(requests, q_heads, dim, dtype=dtype, device=device)
        lists = [self._operators(now, self.one_each, self.qkv, self.heads_out) for now in range(2)]
        scratch = scratch_of(lists[0], device)              # the two never overlap in time
        self.bound = [fc.BoundOperators(ops, scratch) for ops in lists]

    def _operators(self, now, new_tokens, qkv, out=None):
        """A step from state `now` on the queries, keys and values of all new tokens; out: what each request's one new token sees."""
        tokens, (hq, hk, dim) = qkv.shape[0], (self.q_heads, self.kv_heads, self.dim)
        q, k, v = qkv.view(tokens, hq + 2 * hk, dim).split([hq, hk, hk], dim=1)
        of_token = lambda dtype: torch.empty(tokens, dtype=dtype, device=self.device)
        slots, positions = of_token(torch.int64), of_token(torch.int32)
        step = [
            fc.PageMap(page_size=self.page, lengths=self.lengths[now], new_tokens=new_tokens, pool=self.pool, cursor=self.cursor[now], table=self.table,
                       lengths_after=self.lengths[1 - now], row_start=torch.empty(self.requests + 1, dtype=torch.int32, device=self.device), slots=slots,
                       positions=positions, request=of_token(torch.int32), cursor_after=self.cursor[1 - now], unplaced=self.unplaced),
            fc.HeadNormRope(q=q, k=k, v=v, q_out=q, k_cache=self.k_cache, v_cache=self.v_cache, slots=slots, q_weight=self.q_norm, k_weight=self.k_norm,
                            cos_sin=self.angles, positions=positions[None])]
        if out is not None:
            step.append(fc.PagedAttention(q=q, k_cache=self.k_cache, v_cache=self.v_cache, table=self.table, lengths=self.lengths[1 - now], out=out))
        return step

    def admit(self, new_tokens, hidden):
        """new_tokens[r]: prompt tokens that request r adds, or minus its length: it leaves.  hidden: the layer's input for all of
        them, requests in order."""
        new = torch.as_tensor(new_tokens, dtype=torch.int32, device=self.device)
        ops = self._operators(self.now, new, hidden @ self.qkv_weight)
        fc.fc_run_operators(ops, scratch_of(ops, self.device), torch.cuda.current_stream().cuda_stream)
        self.now = 1 - self.now

    def decode(self):
        """A token of every request: self.hidden is its input, and the next step's input when it returns."""
        torch.mm(self.hidden, self.qkv_weight, out=self.qkv)
        self.bound[self.now](torch.cuda.current_stream().cuda_stream)
        torch.mm(self.heads_out.view(self.requests, -1), self.out_weight, out=self.hidden)
        self.now = 1 - self.now

    def graph_of_two(self):
        """Two decoding steps, which lead back to the state they began with, as a graph."""
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.decode()
            self.decode()
        return graph


class HeadNormRopeFunction(torch.autograd.Function):
    """q, k [T, heads, D], norm weights [D], angles as HeadNormRope takes them -> q and k normed and turned.  Differentiable once: backward
    is a kernel itself, and a gradient of it is refused."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos_sin, positions):
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        ops = [fc.HeadNormRope(q=q, k=k, q_out=q_out, k_out=k_out, q_weight=q_weight, k_weight=k_weight, cos_sin=cos_sin, positions=positions)]
        fc.fc_run_operators(ops, scratch_of(ops, q.device), torch.cuda.current_stream().cuda_stream)
        ctx.save_for_backward(q, k, q_weight, k_weight, cos_sin, positions)
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, cos_sin, positions = ctx.saved_tensors
        dq, dk = torch.empty_like(q), torch.empty_like(k)
        dq_weight, dk_weight = (torch.empty(w.shape, dtype=torch.float32, device=w.device) for w in (q_weight, k_weight))
        ops = [fc.HeadNormRopeGrad(q=q, k=k, q_weight=q_weight, k_weight=k_weight, cos_sin=cos_sin, positions=positions, dq_out=dq_out.contiguous(),
                                   dk_out=dk_out.contiguous(), dq=dq, dk=dk, dq_weight=dq_weight, dk_weight=dk_weight)]
        fc.fc_run_operators(ops, scratch_of(ops, q.device), torch.cuda.current_stream().cuda_stream)
        return dq, dk, dq_weight.to(q_weight.dtype), dk_weight.to(k_weight.dtype), None, None


def main():
    p = argparse.ArgumentParser()
    for name, value in (("requests", 64), ("steps", 64), ("q_heads", 32), ("kv_heads", 8), ("dim", 128), ("page", 16), ("prompt", 512)):
        p.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    a = p.parse_args()
    max_len = a.prompt + a.steps + 2
    per_request = -(-max_len // a.page)
    server = Server(a.requests, max_len, a.requests * per_request, a.page, a.q_heads, a.kv_heads, a.dim)
    g = torch.Generator("cpu").manual_seed(1)
    prompts = torch.randint(1, a.prompt + 1, (a.requests,), generator=g)
    width = server.hidden.shape[1]
    tokens = lambda n: torch.randn(n, width, device="cuda").to(server.dtype)
    server.admit(prompts, tokens(int(prompts.sum())))
    server.hidden.copy_(tokens(a.requests))
    # the first request leaves and another comes in its place
    leaves, comes = torch.zeros(a.requests, dtype=torch.int32), torch.zeros(a.requests, dtype=torch.int32)
    leaves[0], comes[0] = -int(prompts[0]), a.prompt
    server.admit(leaves, tokens(0))
    server.admit(comes, tokens(a.prompt))
    server.decode()
    server.decode()
    torch.cuda.synchronize()
    graph = server.graph_of_two()
    begin = time.perf_counter()
    for _ in range(a.steps // 2):
        graph.replay()
    torch.cuda.synchronize()
    if a.steps >= 2:
        seconds = (time.perf_counter() - begin) / (a.steps // 2 * 2)
        print(f"{a.requests} requests, {int(server.lengths[server.now].sum())} tokens in the cache at the end, {int(server.unplaced)} without a page: "
              f"{seconds * 1e6:.1f} us a step with the layer's two products", flush=True)

    # norm weights learnt from the heads they make
    q, k = (torch.randn(256, h, a.dim, device="cuda") for h in (a.q_heads, a.kv_heads))
    cos_sin, positions = angle_table(256, a.dim, "cuda"), torch.arange(256, dtype=torch.int32, device="cuda")[None]
    goal = [w.float() for w in (server.q_norm, server.k_norm)]
    with torch.no_grad():
        goal_q, goal_k = HeadNormRopeFunction.apply(q, k, *goal, cos_sin, positions)
    learnt = [torch.ones(a.dim, device="cuda", requires_grad=True) for _ in goal]
    optimizer = torch.optim.SGD(learnt, lr=0.4 * a.dim)
    for step in range(5):
        out_q, out_k = HeadNormRopeFunction.apply(q, k, *learnt, cos_sin, positions)
        loss = (out_q - goal_q).square().mean() + (out_k - goal_k).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        print(f"training step {step}: loss {float(loss.detach()):.3e}", flush=True)


if __name__ == "__main__":
    main()
