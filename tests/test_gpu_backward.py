"""The layer's gradients around its experts on the GPU against the oracle in 64 bits.

Tolerances: a product or sum of n terms in fp32, in whatever order, is off by at most n 2^-24 times the sum of the terms'
magnitudes (and one step more for each term's own rounding); a result in bfloat16 by 2^-8 of its value besides."""
import sys

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import grad_oracle as go
from hmoe_testlib import to_device, to_host_f32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def hm():
    import paper_2504_05897_amd as hm
    return hm


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


class Problem:
    def __init__(self, hm, dtype, T, H, E, K, seed=0, scale=1.0):
        rng = np.random.default_rng(seed)
        self.bf16 = dtype != "f32"
        kind = {"f32": hm.HMOE_F32, "bf16": hm.HMOE_BF16, "w4": hm.HMOE_BF16_W4, "i8": hm.HMOE_BF16_I8}[dtype]
        self.desc = hm.make_desc(H, 128, E, K, E, kind)
        self.dt = torch.bfloat16 if self.bf16 else torch.float32
        self.step = 2.0 ** -8 if self.bf16 else U
        A = T * K
        store = lambda *s: wl.store((rng.standard_normal(s) * scale).astype(np.float32), wl.BF16 if self.bf16 else wl.F32)
        self.dy, self.o, self.dx_perm, self.x, self.w_g, self.add = (store(*s) for s in ((T, H), (A, H), (A, H), (T, H), (E, H), (T, H)))
        self.idx = np.argsort(rng.standard_normal((T, E)), axis=1)[:, :K].astype(np.int32)
        w = np.exp(rng.standard_normal((T, K)))
        self.w = (w / w.sum(1, keepdims=True)).astype(np.float32)
        self.dw = rng.standard_normal((T, K)).astype(np.float32)
        self.inv = np.empty(A, np.int32)
        self.inv[np.argsort(self.idx.ravel(), kind="stable")] = np.arange(A)
        self.d_logits = rng.standard_normal((T, E)).astype(np.float32)

    def empty(self, *shape, dtype=None):
        return torch.full(shape, float("nan"), dtype=self.dt if dtype is None else dtype, device=DEV)

    def value(self, a):
        return wl.as_f64(a)


SIZES = [("bf16", 1, 8, 1, 1), ("bf16", 1, 2048, 64, 6), ("bf16", 3, 136, 5, 3), ("bf16", 70, 1032, 40, 8), ("bf16", 33, 4104, 9, 2),
         ("bf16", 9, 512, 32, 12), ("f32", 1, 1, 2, 1), ("f32", 7, 37, 8, 2), ("f32", 16, 256, 8, 2), ("f32", 130, 520, 20, 9),
         ("w4", 5, 128, 4, 2), ("i8", 5, 128, 4, 2)]


@pytest.mark.parametrize("dtype,T,H,E,K", SIZES)
def test_combine_backward(hm, dtype, T, H, E, K):
    say("combine backward", dtype, T, H, E, K)
    p = Problem(hm, dtype, T, H, E, K)
    A = T * K
    d_o, d_w = p.empty(A, H), p.empty(T, K, dtype=torch.float32)
    dy, o, inv, w = (to_device(a) for a in (p.dy, p.o, p.inv, p.w))
    hm.hmoe_combine_backward(p.desc, dy, o, inv, w, T, d_o, d_w)
    torch.cuda.synchronize()
    ref_o, ref_w = go.combine_backward(p.value(p.dy), p.value(p.o), p.inv, p.w)
    assert (np.abs(to_host_f32(d_o) - ref_o) <= p.step * np.abs(ref_o) + 2 * U * np.abs(ref_o)).all()
    mags = np.stack([(np.abs(p.value(p.dy)[t]) * np.abs(p.value(p.o)[p.inv[t * K:(t + 1) * K]])).sum(1) for t in range(T)])
    assert (np.abs(to_host_f32(d_w) - ref_w) <= (H + 1) * U * mags).all()
    # one result at a time, and the rows' gradient in the place of the rows: the same bits
    alone_o, alone_w = p.empty(A, H), p.empty(T, K, dtype=torch.float32)
    hm.hmoe_combine_backward(p.desc, dy, None, inv, w, T, alone_o, None)
    hm.hmoe_combine_backward(p.desc, dy, o, inv, None, T, None, alone_w)
    again = p.empty(T, K, dtype=torch.float32)
    hm.hmoe_combine_backward(p.desc, dy, o, inv, w, T, o, again)
    torch.cuda.synchronize()
    for a, b in ((alone_o, d_o), (alone_w, d_w), (o, d_o), (again, d_w)):
        assert torch.equal(a, b)


def test_combine_backward_of_assignments_without_a_row(hm):
    say("combine backward, rows missing")
    p = Problem(hm, "bf16", 6, 64, 4, 2)
    inv = p.inv.copy()
    lost = [inv[3], inv[8]]
    inv[3], inv[8] = -1, 12
    d_o, d_w = torch.full((12, 64), 7.0, dtype=torch.bfloat16, device=DEV), p.empty(6, 2, dtype=torch.float32)
    hm.hmoe_combine_backward(p.desc, to_device(p.dy), to_device(p.o), to_device(inv), to_device(p.w), 6, d_o, d_w)
    torch.cuda.synchronize()
    ref_o, ref_w = go.combine_backward(p.value(p.dy), p.value(p.o), inv, p.w)
    got_o, got_w = to_host_f32(d_o), to_host_f32(d_w)
    assert got_w.ravel()[3] == 0 and got_w.ravel()[8] == 0 and (got_o[lost] == 7.0).all()
    keep = np.setdiff1d(np.arange(12), lost)
    assert (np.abs(got_o[keep] - ref_o[keep]) <= (2.0 ** -8 + 2 * U) * np.abs(ref_o[keep])).all()
    assert np.allclose(got_w, ref_w, atol=1e-3)


@pytest.mark.parametrize("dtype,T,H,E,K", SIZES)
def test_permute_backward(hm, dtype, T, H, E, K):
    say("permute backward", dtype, T, H, E, K)
    p = Problem(hm, dtype, T, H, E, K, seed=1)
    d, inv, add = to_device(p.dx_perm), to_device(p.inv), to_device(p.add)
    mags = np.abs(p.value(p.dx_perm))[p.inv].reshape(T, K, H).sum(1)
    for extra in (None, add):
        dx = p.empty(T, H)
        hm.hmoe_permute_backward(p.desc, d, inv, T, extra, dx)
        torch.cuda.synchronize()
        ref = go.permute_backward(p.value(p.dx_perm), p.inv, T, None if extra is None else p.value(p.add))
        slack = (K + 1) * U * (mags + (0 if extra is None else np.abs(p.value(p.add))))
        assert (np.abs(to_host_f32(dx) - ref) <= p.step * (np.abs(ref) + slack) + slack).all()
    hm.hmoe_permute_backward(p.desc, d, inv, T, add, add)      # in the place of what is added
    torch.cuda.synchronize()
    assert torch.equal(add, dx)


@pytest.mark.parametrize("T,E,K", [(1, 1, 1), (5, 8, 2), (300, 9, 9), (77, 16, 3), (2, 31, 31), (64, 64, 6), (9, 100, 8), (33, 256, 32)])
def test_route_backward(hm, T, E, K):
    say("route backward", T, E, K)
    p = Problem(hm, "bf16", T, 8, E, K, seed=2)
    d = p.empty(T, E, dtype=torch.float32)
    hm.hmoe_route_backward(p.desc, to_device(p.idx), to_device(p.w), to_device(p.dw), T, d)
    torch.cuda.synchronize()
    ref = go.route_backward(p.idx, p.w, p.dw, E)
    largest = np.abs(p.dw).max(1, keepdims=True)               # |dw - mean| <= 2 largest; the mean is a sum of K terms
    assert (np.abs(d.cpu().numpy() - ref) <= 2 * (K + 3) * U * largest * (ref != 0)).all()


def test_route_backward_of_odd_choices(hm):
    """An id that a token names twice gets the sum of both; ids outside the experts are left out."""
    say("route backward, odd ids")
    desc = hm.make_desc(8, 128, 5, 3, 5, hm.HMOE_BF16)
    idx = np.array([[1, 1, 4], [0, -1, 2], [5, 3, 3]], np.int32)
    rng = np.random.default_rng(0)
    w, dw = rng.random((3, 3)).astype(np.float32), rng.standard_normal((3, 3)).astype(np.float32)
    d = torch.full((3, 5), float("nan"), device=DEV)
    hm.hmoe_route_backward(desc, to_device(idx), to_device(w), to_device(dw), 3, d)
    torch.cuda.synchronize()
    assert np.allclose(d.cpu().numpy(), go.route_backward(idx, w, dw, 5), atol=1e-6)


ROUTER = [("bf16", 1, 16, 1, 1), ("bf16", 1, 2048, 64, 6), ("bf16", 17, 144, 5, 3), ("bf16", 200, 1040, 40, 8), ("bf16", 33, 4112, 9, 2),
          ("bf16", 513, 512, 97, 12), ("bf16", 66, 48, 256, 8), ("bf16", 1500, 272, 64, 2), ("f32", 1, 1, 2, 1), ("f32", 7, 37, 8, 2),
          ("f32", 16, 256, 8, 2), ("f32", 700, 130, 67, 9), ("f32", 2100, 36, 33, 2), ("i8", 40, 128, 4, 2)]


@pytest.mark.parametrize("dtype,T,H,E,K", ROUTER)
def test_router_backward(hm, dtype, T, H, E, K):
    say("router backward", dtype, T, H, E, K)
    p = Problem(hm, dtype, T, H, E, K, seed=3)
    x, w_g, d, add = (to_device(a) for a in (p.x, p.w_g, p.d_logits, p.add))
    n = hm.hmoe_router_backward_workspace_bytes(p.desc, T)
    ws = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    xv, wv, dv = p.value(p.x), p.value(p.w_g), p.d_logits.astype(np.float64)
    dx_mags, dw_mags = np.abs(dv) @ np.abs(wv), np.abs(dv).T @ np.abs(xv)
    results = []
    for extra in (None, add):
        dx, d_w = p.empty(T, H), p.empty(E, H, dtype=torch.float32)
        hm.hmoe_router_backward(p.desc, x, w_g, d, T, extra, dx, d_w, ws, n)
        torch.cuda.synchronize()
        ref_dx, ref_dw = go.router_backward(xv, wv, dv, None if extra is None else p.value(p.add))
        slack = (E + 2) * U * (dx_mags + (0 if extra is None else np.abs(p.value(p.add))))
        if p.bf16:
            # the kernel may carry d_logits in two pieces of 8 bits: 2^-17 of each term
            slack = slack + 2.0 ** -17 * dx_mags
        assert (np.abs(to_host_f32(dx) - ref_dx) <= p.step * (np.abs(ref_dx) + slack) + slack).all()
        assert (np.abs(to_host_f32(d_w) - ref_dw) <= (T + 2) * U * dw_mags).all()
        results.append((dx, d_w))
    assert (ws[n:] == 0x5a).all()
    dx, d_w = results[1]
    only_dx, only_dw = p.empty(T, H), p.empty(E, H, dtype=torch.float32)
    hm.hmoe_router_backward(p.desc, None, w_g, d, T, add, only_dx, None, ws, n)
    hm.hmoe_router_backward(p.desc, x, None, d, T, None, None, only_dw, ws, n)
    hm.hmoe_router_backward(p.desc, x, w_g, d, T, add, add, None, ws, n)       # in the place of what is added
    torch.cuda.synchronize()
    assert torch.equal(only_dx, dx) and torch.equal(only_dw, d_w) and torch.equal(add, dx)


def test_router_backward_of_no_tokens_writes_zeros(hm):
    say("router backward, no tokens")
    desc = hm.make_desc(64, 128, 5, 2, 5, hm.HMOE_BF16)
    n = hm.hmoe_router_backward_workspace_bytes(desc, 0)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    d_w = torch.full((5, 64), 7.0, device=DEV)
    hm.hmoe_router_backward(desc, None, None, None, 0, None, None, d_w, ws, n)
    torch.cuda.synchronize()
    assert (d_w == 0).all()


@pytest.mark.parametrize("where", ["x", "d_logits"])
def test_router_backward_carries_infinities_and_nans(hm, where):
    """A value that is not finite reaches the results it takes part in, and no others."""
    say("router backward, not finite", where)
    p = Problem(hm, "bf16", 40, 64, 6, 2, seed=5)
    x, d = p.x.copy(), p.d_logits.copy()
    if where == "x":
        x[7, 3] = 0x7fc0
    else:
        d[7, 2] = np.inf
    n = hm.hmoe_router_backward_workspace_bytes(p.desc, 40)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    dx, d_w = p.empty(40, 64), p.empty(6, 64, dtype=torch.float32)
    hm.hmoe_router_backward(p.desc, to_device(x), to_device(p.w_g), to_device(d), 40, None, dx, d_w, ws, n)
    torch.cuda.synchronize()
    dx, d_w = ~np.isfinite(to_host_f32(dx)), ~np.isfinite(to_host_f32(d_w))
    if where == "x":
        assert not dx.any() and d_w[:, 3].all() and not np.delete(d_w, 3, 1).any()
    else:
        assert dx[7].all() and not np.delete(dx, 7, 0).any() and d_w[2].all() and not np.delete(d_w, 2, 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_in_a_graph(hm, dtype):
    """All four captured together and replayed on new inputs, with eager work in between: the eager results' bits."""
    say("gradients in a graph", dtype)
    T, H, E, K = 600, 256, 24, 4
    p = Problem(hm, dtype, T, H, E, K, seed=6)
    dy, o, inv, w, idx, x, w_g, dxp = (to_device(a) for a in (p.dy, p.o, p.inv, p.w, p.idx, p.x, p.w_g, p.dx_perm))
    n = hm.hmoe_router_backward_workspace_bytes(p.desc, T)

    def chain(ws):
        d_o, d_w, dx = p.empty(T * K, H), p.empty(T, K, dtype=torch.float32), p.empty(T, H)
        d_l, d_wg = p.empty(T, E, dtype=torch.float32), p.empty(E, H, dtype=torch.float32)
        hm.hmoe_combine_backward(p.desc, dy, o, inv, w, T, d_o, d_w)
        hm.hmoe_permute_backward(p.desc, dxp, inv, T, None, dx)
        hm.hmoe_route_backward(p.desc, idx, w, d_w, T, d_l)
        hm.hmoe_router_backward(p.desc, x, w_g, d_l, T, dx, dx, d_wg, ws, n)
        return [d_o, d_w, dx, d_l, d_wg]

    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2)]
    chain(ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain(ws[0])
    for seed in range(3):
        dy.copy_(to_device(Problem(hm, dtype, T, H, E, K, seed=30 + seed).dy))
        graph.replay()
        torch.cuda.synchronize()
        want = chain(ws[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


@pytest.mark.parametrize("dtype,T", [("i8", 5), ("i8", 300), ("bf16", 40), ("f32", 9)])
def test_router_gradient_of_a_layer(hm, dtype, T):
    """A forward pass and the gradient of 1/2 |y - target|^2 with respect to the router, experts held: against the oracle's chain
    over the pass's own choice and expert outputs."""
    say("router gradient", dtype, T)
    bf16 = dtype != "f32"
    shape = wl.small_shape(dtype=wl.BF16 if bf16 else wl.F32, hidden=256, ffn=128, n_experts=8, top_k=2, shared_ffn=(128,), x_mode="rmsnorm")
    lay = wl.make_layer(shape, 7, T)
    kind = {"f32": hm.HMOE_F32, "bf16": hm.HMOE_BF16, "i8": hm.HMOE_BF16_I8}[dtype]
    layer = hm.MoELayer(hm.make_desc(256, 128, 8, 2, 8, kind), lay.experts, lay.shared, lay.w_router, max_tokens=T + 3)
    x = to_device(lay.x)
    y = layer.forward(x)
    target = torch.randn(T, 256, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(y.dtype)
    dy = (y - target).contiguous()
    seen = torch.randn(T, 256, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).to(y.dtype)
    dx = seen.clone()
    d_w, d_logits = layer.router_gradient(x, dy, dx)
    torch.cuda.synchronize()
    f = lambda t: t.double().cpu().numpy()
    idx, w, inv = layer.topk_idx[:T].cpu().numpy(), f(layer.topk_w[:T]), layer.inv_perm[:2 * T].cpu().numpy()
    o = f(layer.o_perm[:2 * T])
    _, d_topk = go.combine_backward(f(dy), o, inv, w)
    ref_l = go.route_backward(idx, w, d_topk, 8)
    ref_dx, ref_w = go.router_backward(f(x), wl.as_f64(lay.w_router), ref_l, f(seen))
    # d_topk_w: 256 products; |d_logits| <= 2 w max |d_topk_w|
    mags = np.stack([(np.abs(f(dy)[t]) * np.abs(o[inv[2 * t:2 * t + 2]])).sum(1) for t in range(T)]).max(1, keepdims=True)
    slack = 2 * (256 + 8) * U * mags * (ref_l != 0)
    assert (np.abs(f(d_logits) - ref_l) <= slack).all()
    xa, wa = np.abs(f(x)), np.abs(wl.as_f64(lay.w_router))
    slack_w = slack.T @ xa + (T + 2) * U * (np.abs(ref_l).T @ xa)
    assert (np.abs(f(d_w) - ref_w) <= slack_w).all()
    slack_x = slack @ wa + ((8 + 2) * U + 2.0 ** -17) * (np.abs(ref_l) @ wa + np.abs(f(seen)))
    assert (np.abs(f(dx) - ref_dx) <= slack_x + (2.0 ** -8 if bf16 else U) * (np.abs(ref_dx) + slack_x)).all()
    # a smaller batch of the same layer, and the layer without an input gradient asked for
    layer.forward(x[:1].contiguous())
    d_w, d_logits = layer.router_gradient(x[:1].contiguous(), dy[:1].contiguous())
    torch.cuda.synchronize()
    assert d_logits.shape == (1, 8) and torch.isfinite(d_w).all()
    layer.close()


def test_router_gradient_captured_with_the_forward_pass(hm):
    """A training step of the router in a graph, replayed as the weights change: int8 experts, gradient, and the eager step's bits."""
    say("router training step in a graph")
    T = 130
    shape = wl.small_shape(dtype=wl.BF16, hidden=256, ffn=128, n_experts=8, top_k=2, x_mode="rmsnorm")
    lay = wl.make_layer(shape, 9, T)
    a, b = (hm.MoELayer(hm.make_desc(256, 128, 8, 2, 8, hm.HMOE_BF16_I8), lay.experts, (), lay.w_router, max_tokens=T) for _ in range(2))
    x = to_device(lay.x)
    dy = torch.randn(T, 256, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).bfloat16()

    def step(layer):
        layer.forward(x)
        return layer.router_gradient(x, dy)

    step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got_w, got_l = step(a)
    for seed in range(3):
        w = a.w_router + 0.01 * torch.randn(8, 256, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).bfloat16()
        a.w_router.copy_(w)
        b.w_router.copy_(w)
        graph.replay()
        torch.cuda.synchronize()
        want_w, want_l = step(b)
        torch.cuda.synchronize()
        assert torch.equal(got_w, want_w) and torch.equal(got_l, want_l), seed
    a.close()
    b.close()


def test_layer_without_a_router(hm):
    say("router gradient, logits from outside")
    shape = wl.small_shape(dtype=wl.BF16, hidden=256, ffn=128, n_experts=8, top_k=2)
    lay = wl.make_layer(shape, 3, 6)
    layer = hm.MoELayer(hm.make_desc(256, 128, 8, 2, 8, hm.HMOE_BF16_I8), lay.experts, (), None, max_tokens=6)
    x, logits = to_device(lay.x), torch.randn(6, 8, device=DEV)
    y = layer.forward(x, logits)
    d_w, d_logits = layer.router_gradient(x, y.clone())
    torch.cuda.synchronize()
    assert d_w is None and d_logits.shape == (6, 8) and torch.isfinite(d_logits).all()
    assert (d_logits.sum(1).abs() <= 1e-5 * d_logits.abs().sum(1) + 1e-12).all()      # softmax does not see a shift of all logits
    layer.close()


@pytest.mark.parametrize("dtype,T,H,E", [("bf16", 2049, 272, 32), ("bf16", 9000, 144, 61), ("bf16", 2500, 1040, 64), ("bf16", 3001, 128, 97),
                                         ("bf16", 2100, 80, 130), ("f32", 2049, 68, 20), ("f32", 5000, 37, 33)])
def test_router_backward_of_large_batches(hm, dtype, T, H, E):
    """Beyond the batches that one launch does: blocks that go from tokens to tokens, chunks of tokens, ends that are no multiples."""
    say("router backward, large", dtype, T, H, E)
    p = Problem(hm, dtype, T, H, E, 1, seed=8)
    x, w_g, d, add = (to_device(a) for a in (p.x, p.w_g, p.d_logits, p.add))
    n = hm.hmoe_router_backward_workspace_bytes(p.desc, T)
    ws = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    dx, d_w = p.empty(T + 1, H), p.empty(E + 1, H, dtype=torch.float32)
    hm.hmoe_router_backward(p.desc, x, w_g, d, T, add, dx, d_w, ws, n)
    torch.cuda.synchronize()
    assert dx[T].isnan().all() and d_w[E].isnan().all() and (ws[n:] == 0x5a).all()
    xv, wv, dv = p.value(p.x), p.value(p.w_g), p.d_logits.astype(np.float64)
    ref_dx, ref_dw = go.router_backward(xv, wv, dv, p.value(p.add))
    slack = ((E + 2) * U + (2.0 ** -17 if p.bf16 else 0)) * (np.abs(dv) @ np.abs(wv)) + 2 * U * np.abs(p.value(p.add))
    assert (np.abs(to_host_f32(dx[:T]) - ref_dx) <= p.step * (np.abs(ref_dx) + slack) + slack).all()
    assert (np.abs(to_host_f32(d_w[:E]) - ref_dw) <= (T + 2) * U * (np.abs(dv).T @ np.abs(xv))).all()
    alone = p.empty(T, H)
    hm.hmoe_router_backward(p.desc, None, w_g, d, T, None, alone, None, ws, n)
    torch.cuda.synchronize()
    ref = go.router_backward(xv, wv, dv)[0]
    assert (np.abs(to_host_f32(alone) - ref) <= p.step * (np.abs(ref) + slack) + slack).all()


@pytest.mark.parametrize("dtype,T,H,K", [("bf16", 6, 64, 2), ("bf16", 7, 72, 11), ("f32", 6, 64, 3), ("f32", 5, 37, 2)])
def test_permute_backward_of_assignments_without_a_row(hm, dtype, T, H, K):
    """An assignment outside [0, T*K) adds nothing, whatever row 0 holds; a token may have none left."""
    say("permute backward, rows missing", dtype, T, H, K)
    p = Problem(hm, dtype, T, H, 16, K, seed=4)
    inv = p.inv.copy()
    inv[K:2 * K] = -1
    inv[-1] = T * K
    rows = np.array(p.value(p.dx_perm))
    rows[p.inv[K:2 * K]] = 0.0
    rows[p.inv[-1]] = 0.0
    ref = go.permute_backward(rows, p.inv, T, None)
    slack = (K + 1) * U * np.abs(rows)[p.inv].reshape(T, K, H).sum(1)
    dx_perm = to_device(p.dx_perm)
    unnamed = sorted({int(r) for r in p.inv[K:2 * K]} | {int(p.inv[-1])})
    dx_perm[unnamed] = float("inf")
    dx = p.empty(T, H)
    hm.hmoe_permute_backward(p.desc, dx_perm, to_device(inv), T, None, dx)
    torch.cuda.synchronize()
    got = to_host_f32(dx)
    assert (np.abs(got - ref) <= p.step * (np.abs(ref) + slack) + slack).all() and (got[1] == 0).all()


@pytest.mark.parametrize("T,H,E", [(40, 144, 3), (300, 272, 40), (2100, 144, 32), (2500, 272, 61), (2100, 128, 97), (2060, 80, 131)])
def test_router_input_gradient_whose_terms_cancel(hm, T, H, E):
    """Three gates per token that sum to zero over router rows with a common value in every column: dx is zero, and what the kernel
    leaves is its own error.  Whole multiples of 2^-22 below 4, so that the values and their sum are exact.  Tolerance: each of the
    three values goes through at most three additions in fp32, each off by one step (2^-23 of at most the sum of magnitudes,
    whichever way it rounds), and zeros add nothing."""
    say("router backward, cancelling", T, H, E)
    desc = hm.make_desc(H, 128, E, 3, E, hm.HMOE_BF16)
    rng = np.random.default_rng(T + E)
    a = np.rint(rng.uniform(-1, 1, (T, 2)) * 2 ** 22) / 2 ** 22
    values = np.concatenate([a, -a.sum(1, keepdims=True)], 1)
    d = np.zeros((T, E), np.float32)
    np.put_along_axis(d, np.argsort(rng.standard_normal((T, E)), axis=1)[:, :3], values.astype(np.float32), 1)
    assert (d.astype(np.float64).sum(1) == 0).all()
    w = np.repeat(wl.store(rng.standard_normal((1, H)).astype(np.float32), wl.BF16), E, 0)
    n = hm.hmoe_router_backward_workspace_bytes(desc, T)
    ws, dx = torch.empty(n, dtype=torch.uint8, device=DEV), torch.full((T, H), float("nan"), dtype=torch.bfloat16, device=DEV)
    hm.hmoe_router_backward(desc, None, to_device(w), to_device(d), T, None, dx, None, ws, n)
    torch.cuda.synchronize()
    mags = np.abs(d).sum(1, keepdims=True).astype(np.float64) * np.abs(wl.as_f64(w)[:1])
    assert (np.abs(to_host_f32(dx)) <= 9 * 2 * U * mags * (1 + 2.0 ** -8)).all()


@pytest.mark.parametrize("dtype,T,H,E", [("bf16", 40, 64, 6), ("bf16", 2100, 144, 30), ("bf16", 2100, 80, 45), ("bf16", 2060, 80, 100),
                                         ("bf16", 2060, 80, 131), ("f32", 40, 37, 6), ("f32", 2060, 36, 21)])
def test_router_backward_of_infinite_gradients(hm, dtype, T, H, E):
    """An infinity of d_logits gives what the sums give: an infinity with the sign of its product, in its token's dx and its expert's
    d_w_g, and a NaN where two of them meet with opposite signs.  (The last expert and the last token stand next to what the kernels
    fill up with.)"""
    say("router backward, infinite gradients", dtype, T, H, E)
    p = Problem(hm, dtype, T, H, E, 2, seed=12)
    xv, wv = p.value(p.x), p.value(p.w_g)
    assert (xv != 0).all() and (wv != 0).all()
    d = p.d_logits.copy()
    at = [(3, 0, np.inf), (7, E - 1, -np.inf), (T - 1, 1, np.inf), (11, 2, np.inf), (11, 4, -np.inf), (20, E - 1, np.inf), (21, 1, -np.inf)]
    for t, e, v in at:
        d[t, e] = v
    n = hm.hmoe_router_backward_workspace_bytes(p.desc, T)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    dx, d_w = p.empty(T, H), p.empty(E, H, dtype=torch.float32)
    hm.hmoe_router_backward(p.desc, to_device(p.x), to_device(p.w_g), to_device(d), T, None, dx, d_w, ws, n)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        ref_dx = np.stack([(d[t].astype(np.float64)[:, None] * wv).sum(0) for t in sorted({t for t, _, _ in at})])
        ref_dw = np.stack([(d[:, e].astype(np.float64)[:, None] * xv).sum(0) for e in sorted({e for _, e, _ in at})])
    assert np.isinf(ref_dx).any() and np.isinf(ref_dw).any() and np.isnan(ref_dx).any() and np.isnan(ref_dw).any()
    dx, d_w = to_host_f32(dx), to_host_f32(d_w)
    assert np.array_equal(dx[sorted({t for t, _, _ in at})], ref_dx, equal_nan=True)
    assert np.array_equal(d_w[sorted({e for _, e, _ in at})], ref_dw, equal_nan=True)
    assert np.isfinite(np.delete(dx, [t for t, _, _ in at], 0)).all() and np.isfinite(np.delete(d_w, [e for _, e, _ in at], 0)).all()


def test_router_gradient_belongs_to_the_last_pass(hm):
    """Refused: before a pass, for another token count than the last pass.  Taken: the last pass's, and that of a captured pass,
    which a replay makes the last one again."""
    say("router gradient, which pass")
    shape = wl.small_shape(dtype=wl.BF16, hidden=256, ffn=128, n_experts=8, top_k=2, x_mode="rmsnorm")
    lay = wl.make_layer(shape, 9, 12)
    layer = hm.MoELayer(hm.make_desc(256, 128, 8, 2, 8, hm.HMOE_BF16_I8), lay.experts, (), lay.w_router, max_tokens=12)
    x = to_device(lay.x)
    dy = torch.randn(12, 256, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).bfloat16()
    with pytest.raises(AssertionError, match="last forward pass"):
        layer.router_gradient(x, dy)
    layer.forward(x)
    want = [v.clone() for v in layer.router_gradient(x, dy)]
    few = x[:5].contiguous()
    layer.forward(few)
    with pytest.raises(AssertionError, match="of 5 tokens, x has 12"):
        layer.router_gradient(x, dy)
    layer.router_gradient(few, dy[:5].contiguous())
    layer.fused = False                                # the separate calls count as well
    layer.forward(x)
    layer.router_gradient(x, dy)
    layer.fused = True
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x)
    for _ in range(2):
        layer.forward(few)
        graph.replay()
        got = layer.router_gradient(x, dy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    layer.close()


@pytest.mark.parametrize("dtype,T,H,K,times", [("bf16", 700, 2048, 6, 4), ("bf16", 500, 2048, 9, 4), ("bf16", 900, 1928, 2, 10),
                                               ("f32", 350, 2052, 6, 4)])
def test_gradients_of_batches_beyond_the_caches(hm, dtype, T, H, K, times):
    """Rows of 64 MiB and more go past the caches.  Every repetition of a batch's tokens, each with rows of its own, has the bits of
    a call over the batch alone, whose kernels keep them."""
    say("gradients past the caches", dtype, T, H, K)
    p = Problem(hm, dtype, T, H, 16, K, seed=14)
    A, elem = T * K, 2 if p.bf16 else 4
    assert A * H * elem < 64 << 20 and (T + A) * H * elem < 64 << 20 <= times * A * H * elem
    dy, o, dxp, inv, w, add = (to_device(a) for a in (p.dy, p.o, p.dx_perm, p.inv, p.w, p.add))
    d_o, d_w, dx = p.empty(A, H), p.empty(T, K, dtype=torch.float32), p.empty(T, H)
    hm.hmoe_combine_backward(p.desc, dy, o, inv, w, T, d_o, d_w)
    hm.hmoe_permute_backward(p.desc, dxp, inv, T, None, dx)
    dx_add = p.empty(T, H)
    hm.hmoe_permute_backward(p.desc, dxp, inv, T, add, dx_add)
    torch.cuda.synchronize()
    first = np.stack([(p.value(p.dy)[t] * p.value(p.o)[p.inv[t * K:(t + 1) * K]]).sum(1) for t in range(9)])
    mags = np.stack([np.abs(p.value(p.dy)[t] * p.value(p.o)[p.inv[t * K:(t + 1) * K]]).sum(1) for t in range(9)])
    assert (np.abs(d_w[:9].cpu().numpy() - first) <= (H + 1) * U * mags).all()

    many = lambda v: v.repeat(times, *[1] * (v.dim() - 1))
    far = (inv[None] + A * torch.arange(times, dtype=torch.int32, device=DEV)[:, None]).view(-1)
    bits = lambda v: v.view(torch.int16 if v.dtype == torch.bfloat16 else torch.int32)
    same = lambda got, want: (bits(got).view(times, *want.shape) == bits(want)).all()
    big_o, big_w = p.empty(times * A, H), p.empty(times * T, K, dtype=torch.float32)
    o_many, dy_many, w_many, dxp_many = many(o), many(dy), many(w), many(dxp)
    hm.hmoe_combine_backward(p.desc, dy_many, o_many, far, w_many, times * T, big_o, big_w)
    only_w = p.empty(times * T, K, dtype=torch.float32)
    hm.hmoe_combine_backward(p.desc, dy_many, o_many, far, None, times * T, None, only_w)
    torch.cuda.synchronize()
    assert same(big_o, d_o) and same(big_w, d_w) and same(only_w, d_w)
    big_o.fill_(float("nan"))
    hm.hmoe_combine_backward(p.desc, dy_many, None, far, w_many, times * T, big_o, None)
    in_place = p.empty(times * T, K, dtype=torch.float32)
    hm.hmoe_combine_backward(p.desc, dy_many, o_many, far, w_many, times * T, o_many, in_place)     # in the place of the rows
    torch.cuda.synchronize()
    assert same(big_o, d_o) and same(o_many, d_o) and same(in_place, d_w)
    big_x, big_add = p.empty(times * T, H), many(add)
    hm.hmoe_permute_backward(p.desc, dxp_many, far, times * T, None, big_x)
    hm.hmoe_permute_backward(p.desc, dxp_many, far, times * T, big_add, big_add)                    # in the place of what is added
    torch.cuda.synchronize()
    assert same(big_x, dx) and same(big_add, dx_add)


@pytest.mark.parametrize("dtype,n_slots", [("i8", 8), ("i8", 3), ("bf16", 5)])
def test_router_gradient_of_a_large_batch_and_a_partial_cache(hm, dtype, n_slots):
    """Beyond the batches whose router gradient is one launch, with experts staged wave by wave: against the oracle's chain over the
    pass's own choice and expert outputs (bounds as in test_router_gradient_of_a_layer, dx's products exact)."""
    say("router gradient, large", dtype, n_slots)
    T, H, E, K = 2300, 256, 8, 2
    shape = wl.small_shape(dtype=wl.BF16, hidden=H, ffn=128, n_experts=E, top_k=K, n_slots=n_slots, x_mode="rmsnorm")
    lay = wl.make_layer(shape, 17, T)
    kind = hm.HMOE_BF16_I8 if dtype == "i8" else hm.HMOE_BF16
    layer = hm.MoELayer(hm.make_desc(H, 128, E, K, n_slots, kind), lay.experts, (), lay.w_router, max_tokens=T)
    x = to_device(lay.x)
    dy = layer.forward(x).clone()                     # the gradient of 1/2 |y|^2
    seen = torch.randn(T, H, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).bfloat16()
    dx = seen.clone()
    d_w, d_logits = layer.router_gradient(x, dy, dx)
    torch.cuda.synchronize()
    assert n_slots == E or layer.last_plan[3] > 1
    f = lambda t: t.double().cpu().numpy()
    idx, w, inv, o = layer.topk_idx.cpu().numpy(), f(layer.topk_w), layer.inv_perm.cpu().numpy(), f(layer.o_perm)
    _, d_topk = go.combine_backward(f(dy), o, inv, w)
    ref_l = go.route_backward(idx, w, d_topk, E)
    ref_dx, ref_w = go.router_backward(f(x), wl.as_f64(lay.w_router), ref_l, f(seen))
    mags = np.abs(f(dy)[:, None] * o[inv].reshape(T, K, H)).sum(2).max(1, keepdims=True)
    slack = 2 * (H + 8) * U * mags * (ref_l != 0)
    assert (np.abs(f(d_logits) - ref_l) <= slack).all()
    xa, wa = np.abs(f(x)), np.abs(wl.as_f64(lay.w_router))
    assert (np.abs(f(d_w) - ref_w) <= slack.T @ xa + (T + 2) * U * (np.abs(ref_l).T @ xa)).all()
    slack_x = slack @ wa + 3 * (E + 2) * 2 * U * (np.abs(ref_l) @ wa + np.abs(f(seen)))    # three pieces of each term, either rounding
    assert (np.abs(f(dx) - ref_dx) <= slack_x + 2.0 ** -8 * (np.abs(ref_dx) + slack_x)).all()
    layer.close()
