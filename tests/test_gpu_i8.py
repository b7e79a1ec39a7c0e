"""Experts in 8-bit integers (HMOE_BF16_I8) on the GPU against the oracle's evaluation in 64 bits.

Tolerance: an output is off by at most the slack that the oracle states for an evaluation in fp32 (codes of h that lie within
2^-10 of a half may be the other whole number) and half a step of bfloat16, 2^-8 of the value."""
import sys

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import i8_oracle as i8
from hmoe_testlib import to_device, to_host_f32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SKINNY, TILED, REFERENCE = 2, 3, 1


@pytest.fixture(scope="module")
def hm():
    import paper_2504_05897_amd as hm
    return hm


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def offsets_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def check_rows(o, x, offsets, experts):
    """o [A, H] against the oracle, expert by expert"""
    o = to_host_f32(o) if isinstance(o, torch.Tensor) else o
    for e, (lo, hi) in enumerate(zip(offsets[:-1], offsets[1:])):
        if hi > lo:
            ref, slack = i8.expert_ffn(wl.as_f64(x[lo:hi]), *(wl.as_f64(m) for m in experts[e]))
            err = np.abs(o[lo:hi] - ref)
            bound = slack + 2.0 ** -8 * (np.abs(ref) + slack)
            assert (err <= bound).all(), (e, float((err - bound).max()), float(np.abs(ref).max()))
            assert np.abs(ref).max() > 1e-3


def make(hm, hidden, ffn, n_experts, top_k, seed, distinct=None, max_tokens=1):
    """A layer whose experts repeat `distinct` different ones."""
    distinct = n_experts if distinct is None else distinct
    shape = wl.small_shape(dtype=wl.BF16, hidden=hidden, ffn=ffn, n_experts=distinct, top_k=1)
    some = wl.make_layer(shape, seed, n_tokens=1).experts
    experts = [some[e % distinct] for e in range(n_experts)]
    d = hm.make_desc(hidden, ffn, n_experts, top_k, n_experts, hm.HMOE_BF16_I8)
    return d, experts, hm.MoELayer(d, experts, (), None, max_tokens=max_tokens, host_copies=False)


def rows_of(seed, n, hidden):
    return wl.store(np.random.default_rng(seed).standard_normal((n, hidden)).astype(np.float32), wl.BF16)


def workspace(hm, d, A):
    """exactly what the call asks for, with a margin behind it that has to stay as it is"""
    n = hm.hmoe_ffn_workspace_bytes(d, A)
    ws = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    return ws, n


def grouped(hm, d, layer, x, offsets, A, path, active=None, o=None, stream=None):
    ws, n = workspace(hm, d, A)
    o = torch.full((A, d.hidden), float("nan"), dtype=torch.bfloat16, device=DEV) if o is None else o
    hm.hmoe_expert_ffn_grouped(d, layer.cache, x, offsets, A, active, o, ws, n, path, stream)
    torch.cuda.synchronize()
    assert (ws[n:] == 0x5a).all()
    return o


@pytest.mark.parametrize("path", [REFERENCE, SKINNY, TILED])
@pytest.mark.parametrize("hidden,ffn,counts", [
    (128, 128, [1]),                              # one row, one K unit in both products
    (256, 128, [3, 0, 7, 1, 40, 0, 9, 2]),        # decode-sized groups and one of several passes
    (128, 384, [33, 1, 0, 0, 70, 5, 8, 32]),      # an odd number of K units; a half-filled column tile
    (1024, 256, [0, 0, 0, 1, 0, 0, 0, 0]),
    (2176, 640, [16, 17, 31]),                    # 17 and 5 K units
    (640, 512, [130, 0, 64, 257]),                # several row tiles with ragged ends
    (256, 4352, [2, 9]),                          # rows of h longer than a block of the quantiser holds at once
])
def test_ffn_i8_paths(hm, path, hidden, ffn, counts):
    say("ffn i8", path, hidden, ffn, counts)
    d, experts, layer = make(hm, hidden, ffn, len(counts), 1, hidden + ffn, distinct=min(3, len(counts)))
    offsets = offsets_of(counts)
    A = int(offsets[-1])
    x = rows_of(5, A, hidden)
    o = grouped(hm, d, layer, to_device(x), to_device(offsets), A, path)
    check_rows(o, x, offsets, experts)
    layer.close()


def test_paths_agree_bit_for_bit(hm):
    """The sums are exact: the decode and the prefill kernels leave the same bits."""
    say("i8 paths agree")
    counts = [1, 0, 5, 32, 30]
    d, experts, layer = make(hm, 768, 896, len(counts), 1, 3)
    offsets = to_device(offsets_of(counts))
    x = to_device(rows_of(2, sum(counts), 768))
    a, b = (grouped(hm, d, layer, x, offsets, sum(counts), p) for p in (SKINNY, TILED))
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    layer.close()


@pytest.mark.parametrize("path", [REFERENCE, SKINNY, TILED])
def test_rows_with_special_values(hm, path):
    """Zeros give zeros; an infinity or a NaN makes its own row NaN and no other; the largest and smallest values count."""
    say("i8 special rows", path)
    d, experts, layer = make(hm, 256, 128, 2, 1, 7)
    x = wl.as_f32(rows_of(1, 40, 256)).copy()
    x[0] = 0
    x[1, 7] = np.inf
    x[2, 255] = -np.inf
    x[3, 0] = np.nan
    x[4] = 0
    x[4, 9] = 1.0                                   # one value in the row
    x[5] *= np.float32(2.0 ** -110)                 # below the smallest amax
    x[6] = np.where(np.arange(256) % 2, 1e-3, 1e-3)  # all alike: every code 127
    bits = wl.store(x, wl.BF16)
    o = to_host_f32(grouped(hm, d, layer, to_device(bits), to_device(offsets_of([20, 20])), 40, path))
    assert (o[0] == 0).all() and np.isnan(o[1:4]).all()
    keep = np.array([i for i in range(40) if not 1 <= i <= 3])
    assert np.isfinite(o[keep]).all()
    for e, rows in ((0, keep[keep < 20]), (1, keep[keep >= 20])):
        ref, slack = i8.expert_ffn(wl.as_f64(bits[rows]), *(wl.as_f64(m) for m in experts[e]))
        # (2^-100: a result that small may be a denormal or zero)
        assert (np.abs(o[rows] - ref) <= slack + 2.0 ** -8 * (np.abs(ref) + slack) + 2.0 ** -100).all()
    layer.close()


@pytest.mark.parametrize("path", [REFERENCE, SKINNY, TILED])
def test_huge_values_do_not_overflow_in_the_quantiser(hm, path):
    """Values near the end of bfloat16's range: 127 v would be infinite.  Weights small enough that h is finite."""
    say("i8 huge", path)
    d = hm.make_desc(128, 128, 1, 1, 1, hm.HMOE_BF16_I8)
    rng = np.random.default_rng(0)
    w = [wl.store((rng.standard_normal((128, 128)) * s).astype(np.float32), wl.BF16) for s in (2.0 ** -126, 2.0 ** -126, 1.0)]
    layer = hm.MoELayer(d, [tuple(w)], (), None, max_tokens=1, host_copies=False)
    x = wl.store((rng.standard_normal((3, 128)) * 6e37).astype(np.float32), wl.BF16)
    o = grouped(hm, d, layer, to_device(x), to_device(offsets_of([3])), 3, path)
    # the gate and up weights lie below 2^-100: their codes are those of amax = 2^-100, as the oracle's are
    check = to_host_f32(o)
    ref, slack = i8.expert_ffn(wl.as_f64(x), *(wl.as_f64(m) for m in w))
    assert np.isfinite(check).all() and (np.abs(check - ref) <= slack + 2.0 ** -8 * (np.abs(ref) + slack) + 2.0 ** -100).all()
    layer.close()


@pytest.mark.parametrize("path", [REFERENCE, SKINNY, TILED])
def test_only_rows_of_active_and_resident_experts_are_written(hm, path):
    say("i8 active", path)
    counts = [4, 9, 0, 40, 2]
    d, experts, layer = make(hm, 256, 256, len(counts), 1, 9)
    offsets = offsets_of(counts)
    A = int(offsets[-1])
    n_rows = A + 37                                  # a caller may only know how many rows there are at most
    x = rows_of(3, A, 256)
    hm.hmoe_cache_evict(layer.cache, 1)
    o = torch.full((A, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    grouped(hm, d, layer, to_device(x), to_device(offsets), n_rows, path, active=[0, 3], o=o)
    got = to_host_f32(o)
    for e, (lo, hi) in enumerate(zip(offsets[:-1], offsets[1:])):
        if e in (0, 3):
            ref, slack = i8.expert_ffn(wl.as_f64(x[lo:hi]), *(wl.as_f64(m) for m in experts[e]))
            assert (np.abs(got[lo:hi] - ref) <= slack + 2.0 ** -8 * (np.abs(ref) + slack)).all()
        else:
            assert (got[lo:hi] == 7.0).all()
    o.fill_(7.0)                                     # every resident expert, one is not
    grouped(hm, d, layer, to_device(x), to_device(offsets), n_rows, path, o=o)
    got = to_host_f32(o)
    assert (got[4:13] == 7.0).all() and (got[:4] != 7.0).any() and (got[13:] != 7.0).any()
    with pytest.raises(hm.HmoeError) as ei:
        grouped(hm, d, layer, to_device(x), to_device(offsets), n_rows, path, active=[1], o=o)
    assert ei.value.status == hm.HMOE_ERR_NOT_RESIDENT
    layer.close()


@pytest.mark.parametrize("path", [0, REFERENCE, SKINNY, TILED])
def test_gather_of_some_assignments(hm, path):
    """The rows a permutation names need not be the first A / K of x.  The same bits as over the gathered rows."""
    say("i8 gather", path)
    d, experts, layer = make(hm, 256, 128, 4, 2, 3, max_tokens=9)
    x = to_device(rows_of(4, 9, 256))
    perm = torch.tensor([17, 3, 12, 5, 16], dtype=torch.int32, device=DEV)
    offsets = torch.tensor([0, 2, 2, 4, 5], dtype=torch.int32, device=DEV)
    ws, n = workspace(hm, d, 5)
    a, b = (torch.full((5, 256), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hm.hmoe_expert_ffn_grouped_gather(d, layer.cache, x, perm, offsets, 5, None, a, ws, n, path)
    hm.hmoe_expert_ffn_grouped(d, layer.cache, x[(perm // 2).long()].contiguous(), offsets, 5, None, b, ws, n, path)
    torch.cuda.synchronize()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and a.isfinite().all()
    layer.close()


def check_layer(layer, lay, y, T):
    idx, w = layer.topk_idx[:T].cpu().numpy(), layer.topk_w[:T].cpu().numpy()
    f64 = lambda experts: [tuple(wl.as_f64(m) for m in e) for e in experts]
    ref, bound = i8.moe_layer(wl.as_f64(lay.x[:T]), idx, w, f64(lay.experts), f64(lay.shared))
    assert (np.abs(to_host_f32(y) - ref) <= bound).all()


@pytest.mark.parametrize("T", [1, 5, 40, 200])
@pytest.mark.parametrize("n_slots", [5, 8])
def test_i8_layer_with_shared_experts(hm, T, n_slots):
    """Whole forward passes: router, routing, FFN (staged where the cache is partial), shared experts, weighted sum."""
    say("i8 layer", T, n_slots)
    shape = wl.small_shape(dtype=wl.BF16, hidden=256, ffn=128, n_experts=8, top_k=2, n_slots=n_slots, shared_ffn=(128, 128),
                           x_mode="rmsnorm")
    lay = wl.make_layer(shape, 40 + T, T)
    d = hm.make_desc(256, 128, 8, 2, n_slots, hm.HMOE_BF16_I8)
    layer = hm.MoELayer(d, lay.experts, lay.shared, lay.w_router, max_tokens=T)
    y = layer.forward(to_device(lay.x))
    torch.cuda.synchronize()
    check_layer(layer, lay, y, T)
    plain = y.clone()
    layer.fused = layer.overlap_shared = layer.merge_shared = False      # the separate calls, the same bits
    assert torch.equal(layer.forward(to_device(lay.x)).view(torch.int16), plain.view(torch.int16))
    layer.close()


def test_i8_expert_ffn_combine_is_the_calls_it_stands_for(hm):
    say("i8 merged combine")
    shape = wl.small_shape(dtype=wl.BF16, hidden=256, ffn=128, n_experts=8, top_k=2, n_slots=8, shared_ffn=(128,), x_mode="rmsnorm")
    lay = wl.make_layer(shape, 4, 3)
    d = hm.make_desc(256, 128, 8, 2, 8, hm.HMOE_BF16_I8)
    layer = hm.MoELayer(d, lay.experts, lay.shared, lay.w_router, max_tokens=3)
    y = layer.forward(to_device(lay.x)).clone()
    bounds = layer._shared_bounds.data_ptr() + 8 * 3
    layer.y.zero_()
    hm.hmoe_expert_ffn_combine(d, layer.cache, to_device(lay.x), layer.perm, layer.inv_perm, layer.topk_w, layer.offsets, 3, layer.o_perm,
                               layer.ffn_ws, layer.ffn_ws_bytes, layer.shared_desc, layer.shared_cache, bounds, layer.o_shared,
                               layer.shared_ws, layer.shared_ws_bytes, layer.y, layer.sync, layer.sync_bytes)
    torch.cuda.synchronize()
    assert torch.equal(layer.y[:3].view(torch.int16), y.view(torch.int16))
    layer.close()


@pytest.mark.parametrize("T", [1, 6, 70])
def test_i8_layer_in_a_graph_and_on_other_streams(hm, T):
    """Captured once, replayed on new inputs with eager calls of another layer in between; and on a stream of its own."""
    say("i8 graph", T)
    shape = wl.small_shape(dtype=wl.BF16, hidden=384, ffn=256, n_experts=6, top_k=2, x_mode="rmsnorm")
    lay = wl.make_layer(shape, 1, T)
    d = hm.make_desc(384, 256, 6, 2, 6, hm.HMOE_BF16_I8)
    layer, other = (hm.MoELayer(d, lay.experts, (), lay.w_router, max_tokens=T) for _ in range(2))
    x = to_device(lay.x)
    layer.forward(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.forward(x)
    side = torch.cuda.Stream()
    for seed in range(4):
        x.copy_(to_device(rows_of(20 + seed, T, 384)))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = other.forward(x)
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), want.view(torch.int16)), seed
    layer.close()
    other.close()


@pytest.mark.parametrize("T", [1, 8])
def test_mixtral_i8_full_size(hm, T):
    """Large experts as a decode loop uses them: the wide matrices' weight stream, rows of 14336 values of h."""
    say("mixtral i8", T)
    shape = wl.SHAPES["mixtral"]
    lay = wl.make_layer(shape, 1, T, threads=16)
    d = hm.make_desc(shape.hidden, shape.ffn, shape.n_experts, shape.top_k, shape.n_experts, hm.HMOE_BF16_I8)
    layer = hm.MoELayer(d, lay.experts, (), lay.w_router, max_tokens=T, host_copies=False)
    y = layer.forward(to_device(lay.x))
    torch.cuda.synchronize()
    idx, w = layer.topk_idx[:T].cpu().numpy(), layer.topk_w[:T].cpu().numpy()
    named = sorted(set(idx[:1].ravel()))                       # the first token's experts: the oracle takes a while
    ref, bound = i8.moe_layer(wl.as_f64(lay.x[:1]), np.searchsorted(named, idx[:1]), w[:1],
                              [tuple(wl.as_f64(m) for m in lay.experts[e]) for e in named])
    assert (np.abs(to_host_f32(y[:1]) - ref) <= bound).all()
    layer.close()


def test_a_prefill_batch_of_many_tiles(hm):
    """More rows per expert than any tile has, skewed: the first expert takes half of them."""
    say("i8 many tiles")
    counts = [1100, 0, 300, 513, 1, 77, 128, 31]
    d, experts, layer = make(hm, 768, 384, len(counts), 1, 11, distinct=2)
    offsets = offsets_of(counts)
    A = int(offsets[-1])
    x = rows_of(6, A, 768)
    o = grouped(hm, d, layer, to_device(x), to_device(offsets), A, 0)
    check_rows(o, x, offsets, experts)
    again = grouped(hm, d, layer, to_device(x), to_device(offsets), A, 0)
    assert torch.equal(o.view(torch.int16), again.view(torch.int16))
    layer.close()


@pytest.mark.parametrize("tiles", ["00", "11", "22", "33", "44", "55"])
@pytest.mark.parametrize("hidden,ffn,counts", [
    (768, 896, [700, 1, 0, 224, 225, 31]),       # 6 and 7 K steps: an even and an odd number, the fewest of walking blocks
    (896, 1152, [97, 300, 448, 33, 64, 0]),      # 7 and 9
    (1024, 1408, [130] * 9),                     # 8 and 11
    (2304, 768, [256, 129]),                     # 18 and 6
])
def test_every_tile_shape(hm, monkeypatch, tiles, hidden, ffn, counts):
    """Each tile shape of the prefill kernels, with and without weights that pass the caches; the same bits from all of them."""
    say("i8 tiles", tiles, hidden, ffn, counts)
    d, experts, layer = make(hm, hidden, ffn, len(counts), 1, hidden, distinct=2)
    offsets = offsets_of(counts)
    A = int(offsets[-1])
    x = rows_of(8, A, hidden)
    args = (hm, d, layer, to_device(x), to_device(offsets), A, TILED)
    want = grouped(*args)
    monkeypatch.setenv("HMOE_I8_TILES", tiles)
    got = grouped(*args)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    some = np.r_[0:8, A - 8:A]                     # (the oracle: a few rows of the first and the last expert with rows)
    own = np.concatenate([np.full(n, e) for e, n in enumerate(counts)])[some]
    for e in set(own):
        ref, slack = i8.expert_ffn(wl.as_f64(x[some[own == e]]), *(wl.as_f64(m) for m in experts[e]))
        err = np.abs(to_host_f32(got)[some[own == e]] - ref)
        assert (err <= slack + 2.0 ** -8 * (np.abs(ref) + slack)).all()
    layer.close()


def test_walking_blocks_with_many_tiles_each(hm, monkeypatch):
    """Hundreds of tiles of mixed heights: every block of the launch goes through several, in both halves of its weight ring."""
    say("i8 walk, many tiles")
    counts = [40, 300, 224, 500, 97, 161, 193, 1000] * 4
    d, experts, layer = make(hm, 896, 2688, len(counts), 1, 5, distinct=1)
    x = to_device(rows_of(9, sum(counts), 896))
    args = (hm, d, layer, x, to_device(offsets_of(counts)), sum(counts), TILED)
    monkeypatch.setenv("HMOE_I8_TILES", "00")
    want = grouped(*args)
    monkeypatch.setenv("HMOE_I8_TILES", "22")
    for _ in range(3):
        assert torch.equal(grouped(*args).view(torch.int16), want.view(torch.int16))
    layer.close()


@pytest.mark.parametrize("T,far", [(4500, False), (6500, True)])
def test_codes_once_per_token(hm, T, far):
    """A batch large enough for one row of codes per token.  The same bits as over the gathered rows, and for a call over some of
    the assignments, whose permutation names tokens past A / K, too."""
    say("i8 codes per token", T, far)
    H, E, K = 1024, 7, 2
    d, experts, layer = make(hm, H, 896, E, K, 13, distinct=2)
    rng = np.random.default_rng(17)
    idx = np.argsort(rng.standard_normal((T, E)), axis=1)[:, :K]
    perm = np.argsort(idx.ravel(), kind="stable").astype(np.int32)
    keep = np.ones(T * K, bool)
    if far:                                          # the assignments of two experts are left out, and some tokens altogether
        keep = ~np.isin(idx.ravel()[perm], [2, 3]) & (perm // K % 97 != 0)
    perm = perm[keep]
    offsets = offsets_of(np.bincount(idx.ravel()[perm], minlength=E))
    A = len(perm)
    assert A * H >= 8 << 20 and (not far or (perm // K >= -(-A // K)).any())
    # (tokens that the permutation does not name hold NaN: nothing may come of them)
    x = np.full((T, H), 0x7fc0, np.uint16)
    named = np.unique(perm // K)
    x[named] = rows_of(12, len(named), H)
    x, perm, offsets = to_device(x), to_device(perm), to_device(offsets)
    ws, n = workspace(hm, d, A)
    a, b = (torch.full((A, H), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for seed in range(2):                            # the second time over a workspace full of the first one's notes
        hm.hmoe_expert_ffn_grouped_gather(d, layer.cache, x, perm, offsets, A, None, a, ws, n, TILED)
        hm.hmoe_expert_ffn_grouped(d, layer.cache, x[(perm // K).long()].contiguous(), offsets, A, None, b, torch.empty_like(ws), n, TILED)
        torch.cuda.synchronize()
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and a.isfinite().all() and (ws[n:] == 0x5a).all()
    layer.close()


def test_large_batch_through_a_partial_cache_and_a_graph(hm):
    """A batch whose tokens are quantised once each: with half of the experts staged wave by wave, and captured and replayed, the
    bits of an eager call with every expert resident."""
    say("i8 large batch, partial cache, graph")
    T, H, F, E, K = 4300, 1024, 256, 8, 2
    shape = wl.small_shape(dtype=wl.BF16, hidden=H, ffn=F, n_experts=E, top_k=K, x_mode="rmsnorm")
    lay = wl.make_layer(shape, 21, T)
    assert T * K * H >= 8 << 20
    whole = hm.MoELayer(hm.make_desc(H, F, E, K, E, hm.HMOE_BF16_I8), lay.experts, (), lay.w_router, max_tokens=T)
    half = hm.MoELayer(hm.make_desc(H, F, E, K, 3, hm.HMOE_BF16_I8), lay.experts, (), lay.w_router, max_tokens=T)
    x = to_device(lay.x)
    want = whole.forward(x).clone()
    got = half.forward(x)
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int16), want.view(torch.int16)) and half.last_plan[3] > 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = whole.forward(x)
    for seed in range(2):
        x.copy_(to_device(rows_of(40 + seed, T, H)))
        graph.replay()
        torch.cuda.synchronize()
        replayed = y.clone()
        assert torch.equal(replayed.view(torch.int16), whole.forward(x).view(torch.int16)), seed
    idx, w = whole.topk_idx[:4].cpu().numpy(), whole.topk_w[:4].cpu().numpy()
    f64 = [tuple(wl.as_f64(m) for m in e) for e in lay.experts]
    ref, bound = i8.moe_layer(wl.as_f64(rows_of(41, T, H)[:4]), idx, w, f64)
    assert (np.abs(to_host_f32(y[:4]) - ref) <= bound).all()
    whole.close()
    half.close()


def test_two_calls_at_once(hm):
    """Two layers' calls on two streams, each with a workspace of its own, again and again: nothing is shared."""
    say("i8 two calls at once")
    counts = [200, 90, 0, 300]
    made = [make(hm, 512, 384, 4, 1, seed, distinct=2) for seed in (31, 32)]
    xs = [to_device(rows_of(50 + i, sum(counts), 512)) for i in range(2)]
    offsets = to_device(offsets_of(counts))
    A = sum(counts)
    want = [grouped(hm, d, layer, x, offsets, A, TILED) for (d, _, layer), x in zip(made, xs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    n = hm.hmoe_ffn_workspace_bytes(made[0][0], A)
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [[torch.empty_like(want[0]) for _ in range(6)] for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(6):
        for i, (d, _, layer) in enumerate(made):
            hm.hmoe_expert_ffn_grouped(d, layer.cache, xs[i], offsets, A, None, outs[i][k], ws[i], n, TILED, streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o.view(torch.int16), want[i].view(torch.int16))
    for _, _, layer in made:
        layer.close()


@pytest.mark.parametrize("tiles", ["06", "07"])
@pytest.mark.parametrize("hidden,ffn,counts", [(640, 512, [1, 160, 161, 0, 320, 33]), (128, 4608, [130, 97, 64]), (1152, 1024, [31, 500, 0, 128])])
def test_down_in_two_halves_of_k(hm, monkeypatch, tiles, hidden, ffn, counts):
    """Two sets of waves per tile (2, 18 and 4 K steps each): the bits of the other tile shapes."""
    say("i8 split", tiles, hidden, ffn, counts)
    d, experts, layer = make(hm, hidden, ffn, len(counts), 1, hidden, distinct=2)
    A = sum(counts)
    args = (hm, d, layer, to_device(rows_of(14, A, hidden)), to_device(offsets_of(counts)), A, TILED)
    monkeypatch.setenv("HMOE_I8_TILES", "00")
    want = grouped(*args)
    monkeypatch.setenv("HMOE_I8_TILES", tiles)
    assert torch.equal(grouped(*args).view(torch.int16), want.view(torch.int16))
    layer.close()


@pytest.mark.parametrize("hidden,ffn", [(128, 14336), (14336, 128)])
def test_codes_beyond_32_bits_of_offset(hm, hidden, ffn):
    """More than 4 GiB of codes (of h, of tokens): every repetition of the same rows has the bits of a call over one of them."""
    say("i8 far rows", hidden, ffn)
    n, times = 1009, 308
    assert n * times * 14336 > 1 << 32
    d, experts, layer = make(hm, hidden, ffn, 1, 1, 21)
    x = to_device(rows_of(15, n, hidden))
    want = grouped(hm, d, layer, x, to_device(offsets_of([n])), n, TILED)
    A = n * times
    o = grouped(hm, d, layer, x.repeat(times, 1), to_device(offsets_of([A])), A, TILED)
    assert (o.view(torch.int16).view(times, n, hidden) == want.view(torch.int16)).all()
    layer.close()


@pytest.mark.parametrize("path", [SKINNY, TILED])
@pytest.mark.parametrize("ffn,rows", [(1408, 2900), (4096, 1100), (4608, 900)])     # rows by waves (two sizes) and by blocks
def test_codes_of_h_are_those_of_the_division(hm, path, ffn, rows):
    """Each code of h is rint(127 h / amax) of the h at hand in fp32, halves and their neighbours included.  (The call's workspace
    holds h first and behind it, at a multiple of 256 bytes, its codes.)"""
    say("i8 codes of h", path, ffn, rows)
    d, experts, layer = make(hm, 128, ffn, 1, 1, 23)
    x, offsets = to_device(rows_of(16, rows, 128)), to_device(offsets_of([rows]))
    n = hm.hmoe_ffn_workspace_bytes(d, rows)
    ws, o = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.empty(rows, 128, dtype=torch.bfloat16, device=DEV)
    hm.hmoe_expert_ffn_grouped(d, layer.cache, x, offsets, rows, None, o, ws, n, path)
    torch.cuda.synchronize()
    at = -(-rows * ffn * 4 // 256) * 256
    h = ws[:rows * ffn * 4].view(torch.float32).view(rows, ffn).cpu().numpy()
    codes = ws[at:at + rows * ffn].view(torch.int8).view(rows, ffn).cpu().numpy()
    amax = np.abs(h).max(1, keepdims=True)
    assert amax.min() > 1e-3 and np.isfinite(h).all()
    want = np.rint(h * np.float32(127) / amax)
    assert want.dtype == np.float32 and (codes == want).all(), int((codes != want).sum())
    layer.close()


@pytest.mark.parametrize("path", [REFERENCE, SKINNY, TILED])
@pytest.mark.parametrize("rows", [2, 40])                    # (two rows: the decode blocks quantise them themselves)
@pytest.mark.parametrize("hidden,ffn,gate_up_std,down_std", [
    (128, 128, 2.0 ** -98, 1.0),              # tokens near the end of the range, h of 2^60
    (4224, 128, 2.0 ** -98, 1.0),             # rows that a whole block quantises
    (128, 128, 2.0 ** -68, 2.0 ** -20),       # h above 2^100 as well: 127 h would be infinite
    (128, 4224, 2.0 ** -68, 2.0 ** -20),
])
def test_codes_of_rows_above_2_to_the_100(hm, path, rows, hidden, ffn, gate_up_std, down_std):
    """Rows whose 127 v is beyond fp32, of tokens and of h, under weights whose codes are not zero."""
    say("i8 rows above 2^100", path, rows, hidden, ffn)
    rng = np.random.default_rng(hidden + ffn)
    draw = lambda std, *s: wl.store((rng.standard_normal(s) * std).astype(np.float32), wl.BF16)
    w = draw(gate_up_std, ffn, hidden), draw(gate_up_std, ffn, hidden), draw(down_std, hidden, ffn)
    layer = hm.MoELayer(hm.make_desc(hidden, ffn, 1, 1, 1, hm.HMOE_BF16_I8), [w], (), None, max_tokens=1, host_copies=False)
    x = draw(6e37, rows, hidden)
    assert np.isfinite(wl.as_f64(x)).all() and 127 * np.abs(wl.as_f64(x)).max() > np.finfo(np.float32).max
    o = to_host_f32(grouped(hm, layer.desc, layer, to_device(x), to_device(offsets_of([rows])), rows, path))
    with np.errstate(over="ignore"):
        ref, slack = i8.expert_ffn(wl.as_f64(x), *(wl.as_f64(m) for m in w))
    assert np.abs(ref).max() > 2.0 ** 60 and np.isfinite(o).all()
    assert (np.abs(o - ref) <= slack + 2.0 ** -8 * (np.abs(ref) + slack)).all()
    layer.close()


@pytest.mark.parametrize("ffn,rows,path", [(2048, 95, TILED), (2048, 96, TILED), (2048, 200, TILED), (2048, 300, 0), (2176, 200, TILED),
                                           (1920, 200, TILED), (2560, 1000, 0)])
def test_down_launches_around_the_rule_for_halves_of_k(hm, ffn, rows, path):
    """What the prefill kernels choose by themselves for one expert: a long F in multiples of four K steps and 96 rows take two
    sets of waves per tile, fewer rows and other lengths do not."""
    say("i8 split rule", ffn, rows, path)
    d, experts, layer = make(hm, 256, ffn, 1, 1, 27)
    x = rows_of(18, rows, 256)
    o = to_host_f32(grouped(hm, d, layer, to_device(x), to_device(offsets_of([rows])), rows, path))
    some = np.unique(np.r_[0:4, rows // 2:rows // 2 + 4, rows - 4:rows])
    check_rows(o[some], x[some], offsets_of([len(some)]), experts)
    assert np.isfinite(o).all()
    layer.close()


@pytest.mark.parametrize("path", [REFERENCE, SKINNY, TILED])
@pytest.mark.parametrize("counts", [[4, 9, 0, 40, 2], [1, 2, 1, 0, 1]])        # (the second: rows quantised by the decode blocks)
def test_every_resident_expert_where_one_is_not(hm, path, counts):
    """A call over all experts, one of them evicted: the others' rows are right, its own and those behind the last stay as they are."""
    say("i8 one expert not resident", path, counts)
    d, experts, layer = make(hm, 256, 256, len(counts), 1, 9)
    offsets = offsets_of(counts)
    A, n_rows = int(offsets[-1]), int(offsets[-1]) + 5
    x = rows_of(3, A, 256)
    hm.hmoe_cache_evict(layer.cache, 1)
    o = torch.full((n_rows, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    x_dev = torch.cat([to_device(x), torch.full((5, 256), float("nan"), dtype=torch.bfloat16, device=DEV)])
    grouped(hm, d, layer, x_dev, to_device(offsets), n_rows, path, o=o)
    got, resident = to_host_f32(o), [0 if e == 1 else n for e, n in enumerate(counts)]
    keep = np.concatenate([np.arange(offsets[e], offsets[e + 1]) for e in range(len(counts)) if e != 1])
    check_rows(got[keep], x[keep], offsets_of(resident), experts)
    assert (np.delete(got, keep, 0) == 7.0).all()
    layer.close()
