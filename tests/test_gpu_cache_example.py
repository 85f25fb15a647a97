"""The example that runs the operators of the paged cache together (examples/cache_operators.py)."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("cache_operators", os.path.join(ROOT, "examples", "cache_operators.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_requests_come_decode_and_leave(example):
    """Every step's attention against the same tokens' in 64 bits, whatever pages they lie on.

    Tolerance: a score is at most sqrt(D) times the norm weights' product (below 2), so below 16 for D = 64, and its 64 products and the norms
    are off by at most about 100 * 2^-24 of that, 1e-4; a weight by that relative, and the output by twice it times the largest value."""
    import torch
    hq, hk, dim, requests = 6, 3, 64, 5
    server = example.Server(requests, 200, 40, page=8, q_heads=hq, kv_heads=hk, dim=dim, width=48, dtype=torch.float32, seed=3)
    g = torch.Generator("cuda").manual_seed(4)
    norm = [w.double().cpu().numpy() for w in (server.q_norm, server.k_norm)]
    angles = server.angles.double().cpu().numpy()
    rows = [[] for _ in range(requests)]                  # the new tokens' queries, keys and values as the layer gave them

    def turned(x, weight, position):
        y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + 1e-6) * weight
        a, b = y[..., :dim // 2], y[..., dim // 2:]
        c, s = angles[position, :dim // 2], angles[position, dim // 2:]
        return np.concatenate((a * c - b * s, b * c + a * s), axis=-1)

    def enter(counts, hidden):
        qkv = (hidden @ server.qkv_weight).double().cpu().numpy().reshape(-1, hq + 2 * hk, dim)
        at = 0
        for r, n in enumerate(counts):
            if n < 0:
                rows[r] = rows[r][:n]
            for _ in range(max(n, 0)):
                rows[r].append(qkv[at])
                at += 1

    def admit(counts):
        hidden = torch.randn(sum(max(n, 0) for n in counts), 48, generator=g, device="cuda")
        enter(counts, hidden)
        server.admit(counts, hidden)

    def decode():
        enter([1] * requests, server.hidden.clone())
        server.decode()
        got = server.heads_out.double().cpu().numpy()
        for r in range(requests):
            x = np.stack(rows[r])
            q = turned(x[-1, :hq], norm[0], len(x) - 1)
            k = np.stack([turned(x[j, hq:hq + hk], norm[1], j) for j in range(len(x))])
            v = x[:, hq + hk:]
            for h in range(hq):
                s = k[:, h // (hq // hk)] @ q[h] * dim ** -0.5
                w = np.exp(s - s.max())
                want = w @ v[:, h // (hq // hk)] / w.sum()
                assert np.abs(got[r, h] - want).max() <= 2e-4 * np.abs(v).max(), (r, h)
        assert server.lengths[server.now].cpu().tolist() == [len(x) for x in rows]

    admit([17, 1, 8, 60, 0])
    server.hidden.normal_(generator=g)
    for _ in range(9):
        decode()
    admit([-26, 0, -3, 0, 0])                             # one leaves, one is cut back
    admit([33, 0, 5, 0, 100])
    for _ in range(4):
        decode()
    assert int(server.unplaced) == 0
    held = server.table.cpu().numpy()
    lengths = server.lengths[server.now].cpu().numpy()
    pages = np.concatenate([held[r, :-(-n // 8)] for r, n in enumerate(lengths)])
    assert len(set(pages.tolist())) == len(pages)         # no page is in two hands


def test_a_graph_of_steps_gives_what_the_steps_give(example):
    import torch
    make = lambda: example.Server(7, 120, 60, page=16, q_heads=8, kv_heads=2, dim=128, width=64, seed=5)
    servers = [make(), make()]
    prompts = torch.tensor([3, 40, 16, 1, 0, 90, 17], dtype=torch.int32)
    g = torch.Generator("cuda").manual_seed(6)
    hidden = torch.randn(int(prompts.sum()), 64, generator=g, device="cuda").bfloat16()
    first = torch.randn(7, 64, generator=g, device="cuda").bfloat16()
    for s in servers:
        s.admit(prompts, hidden)
        s.hidden.copy_(first)
        s.decode()
        s.decode()
        s.decode()
    torch.cuda.synchronize()
    eager, other = servers
    graph = other.graph_of_two()
    for _ in range(4):
        graph.replay()
        eager.decode()
        eager.decode()
        torch.cuda.synchronize()
        assert torch.equal(eager.hidden, other.hidden) and bool(torch.isfinite(eager.hidden).all())
        assert torch.equal(eager.lengths[eager.now], other.lengths[other.now])


def test_the_function_has_the_gradient_of_the_formula(example):
    """Against autograd of the formula in 64 bits.  dq and dk: rows of 48 elements, about 60 roundings of values of order 4, 60 * 2^-24 * 16 = 6e-5
    at most; the weights' gradients are sums of 33 * heads such terms."""
    import torch
    g = torch.Generator("cuda").manual_seed(7)
    q, k = (torch.randn(33, h, 48, generator=g, device="cuda") for h in (5, 2))
    weights = [1 + 0.2 * torch.randn(48, generator=g, device="cuda") for _ in range(2)]
    dy = [torch.randn(x.shape, generator=g, device="cuda") for x in (q, k)]
    cos_sin = example.angle_table(50, 48, "cuda")
    positions = torch.randint(0, 50, (1, 33), generator=g, device="cuda", dtype=torch.int32)

    here = [x.clone().requires_grad_() for x in (q, k, *weights)]
    torch.autograd.backward(example.HeadNormRopeFunction.apply(*here, cos_sin, positions), dy)

    there = [x.double().requires_grad_() for x in (q, k, *weights)]
    c, s = cos_sin.double()[positions[0].long()][:, None].split(24, dim=-1)

    def formula(x, weight):
        y = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight
        a, b = y.split(24, dim=-1)
        return torch.cat((a * c - b * s, b * c + a * s), dim=-1)

    torch.autograd.backward([formula(there[0], there[2]), formula(there[1], there[3])], [d.double() for d in dy])
    for x, y, n in zip(here, there, (1, 1, 33 * 5, 33 * 2)):
        assert float((x.grad.double() - y.grad).abs().max()) <= 6e-5 * n


def test_a_gradient_of_the_function_s_gradient_is_refused(example):
    # backward is not made of differentiable steps: without the refusal the sum's gradient would come out as that of its second term alone
    import torch
    q, k = (torch.randn(5, h, 16, device="cuda", requires_grad=True) for h in (2, 1))
    weights = [torch.ones(16, device="cuda", requires_grad=True) for _ in range(2)]
    out_q, _ = example.HeadNormRopeFunction.apply(q, k, *weights, example.angle_table(9, 16, "cuda"), torch.zeros((1, 5), dtype=torch.int32, device="cuda"))
    slope, = torch.autograd.grad(out_q.square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (slope.square().sum() + q.square().sum()).backward()
