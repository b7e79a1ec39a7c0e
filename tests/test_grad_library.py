"""The layer's gradients around its experts: the oracle against differences, and what the library refuses.  No GPU."""
import ctypes

import numpy as np
import pytest

from oracle import grad_oracle as go


@pytest.fixture(scope="module")
def hm():
    import paper_2504_05897_amd as hm
    return hm


def test_oracle_gradients_are_the_differences_of_the_layer():
    """The chain dy -> d_topk_w -> d_logits -> (dx, d_w_g) and dy -> d_o_perm against central differences of
    L = sum(dy * y), y = sum_j w_j o_j, w = softmax(chosen logits), logits = x W_g^T with the choice held."""
    rng = np.random.default_rng(1)
    T, H, E, K = 4, 6, 5, 3
    x, w_g, dy = rng.standard_normal((T, H)), rng.standard_normal((E, H)), rng.standard_normal((T, H))
    o, idx = rng.standard_normal((T * K, H)), np.argsort(-(x @ w_g.T), axis=1)[:, :K]
    inv = rng.permutation(T * K)

    def gates(x, w_g):
        l = np.take_along_axis(x @ w_g.T, idx, 1)
        p = np.exp(l - l.max(1, keepdims=True))
        return p / p.sum(1, keepdims=True)

    def loss(x, w_g, o):
        return (dy * (gates(x, w_g)[:, :, None] * o[inv].reshape(T, K, H)).sum(1)).sum()

    w = gates(x, w_g)
    d_o, d_w = go.combine_backward(dy, o, inv, w)
    d_logits = go.route_backward(idx, w, d_w, E)
    dx, d_w_g = go.router_backward(x, w_g, d_logits)
    for at, grad in ((0, dx), (1, d_w_g), (2, d_o)):
        args = [x, w_g, o]
        num = np.zeros_like(args[at])
        for i in np.ndindex(*num.shape):
            lo, hi = ([a.copy() for a in args] for _ in range(2))
            lo[at][i] -= 1e-5
            hi[at][i] += 1e-5
            num[i] = (loss(*hi) - loss(*lo)) / 2e-5
        assert np.allclose(grad, num, atol=1e-8), at
    # the gather x_perm[p] = x[t of p]: L = sum(d * x_perm)
    d = rng.standard_normal((T * K, H))
    num = np.zeros((T, H))
    for t in range(T):
        for j in range(K):
            num[t] += d[inv[t * K + j]]
    assert np.allclose(go.permute_backward(d, inv, T, add=dy), num + dy)


def test_bad_arguments_are_refused_on_the_host(hm):
    lib, ok = hm._lib, hm.make_desc(64, 64, 8, 2, 8, hm.HMOE_BF16)
    a = [4096 * (i + 1) for i in range(8)]   # addresses the host only looks at
    by, BAD = ctypes.byref, hm.HMOE_ERR_INVALID_ARG
    bad_desc = hm.make_desc(64, 64, 8, 9, 8, hm.HMOE_BF16)
    odd = hm.make_desc(60, 64, 8, 2, 8, hm.HMOE_BF16)
    eight = hm.make_desc(72, 64, 8, 2, 8, hm.HMOE_BF16)
    combine, permute, route, router = (lib.hmoe_combine_backward, lib.hmoe_permute_backward, lib.hmoe_route_backward,
                                       lib.hmoe_router_backward)
    assert combine(None, *a[:4], 4, a[4], a[5], None) == BAD
    assert combine(by(bad_desc), *a[:4], 4, a[4], a[5], None) == BAD
    assert combine(by(ok), *a[:4], -1, a[4], a[5], None) == BAD
    assert combine(by(ok), *a[:4], 1 << 30, a[4], a[5], None) == BAD                 # T * K beyond 31 bits
    assert combine(by(ok), *a[:4], 4, None, None, None) == BAD                       # neither result
    assert combine(by(ok), None, *a[1:4], 4, a[4], a[5], None) == BAD                # no dy
    assert combine(by(ok), a[0], None, a[2], a[3], 4, None, a[5], None) == BAD       # d_topk_w without o_perm
    assert combine(by(ok), a[0], a[1], a[2], None, 4, a[4], None, None) == BAD       # d_o_perm without topk_w
    assert combine(by(ok), a[0] + 8, *a[1:4], 4, a[4], a[5], None) == BAD            # misaligned rows
    assert combine(by(ok), *a[:4], 4, a[4] + 2, a[5], None) == BAD
    assert combine(by(ok), *a[:4], 4, a[4], a[5] + 2, None) == BAD
    assert combine(by(odd), *a[:4], 4, a[4], a[5], None) == hm.HMOE_ERR_UNSUPPORTED
    assert combine(by(ok), None, None, None, None, 0, None, None, None) == hm.HMOE_OK
    assert permute(by(ok), a[0], a[1], -1, None, a[2], None) == BAD
    assert permute(by(ok), None, a[1], 4, None, a[2], None) == BAD
    assert permute(by(ok), a[0], a[1], 4, None, None, None) == BAD
    assert permute(by(ok), a[0], a[1], 4, a[3] + 4, a[2], None) == BAD
    assert permute(by(odd), a[0], a[1], 4, None, a[2], None) == hm.HMOE_ERR_UNSUPPORTED
    assert permute(by(ok), None, None, 0, None, None, None) == hm.HMOE_OK
    assert route(by(ok), a[0], a[1], a[2], -1, a[3], None) == BAD
    assert route(by(ok), a[0], a[1], None, 4, a[3], None) == BAD
    assert route(by(ok), a[0] + 1, a[1], a[2], 4, a[3], None) == BAD
    assert route(by(ok), None, None, None, 0, None, None) == hm.HMOE_OK
    need = hm.hmoe_router_backward_workspace_bytes(ok, 4)
    assert need > 0 and lib.hmoe_router_backward_workspace_bytes(by(bad_desc), 4) == 0
    assert lib.hmoe_router_backward_workspace_bytes(by(ok), -1) == 0
    assert router(by(ok), a[0], a[1], a[2], -1, None, a[3], a[4], a[5], need, None) == BAD
    assert router(by(ok), a[0], a[1], a[2], 4, None, None, None, a[5], need, None) == BAD     # neither result
    assert router(by(ok), None, a[1], a[2], 4, None, a[3], a[4], a[5], need, None) == BAD     # d_w_g without x
    assert router(by(ok), a[0], None, a[2], 4, None, a[3], a[4], a[5], need, None) == BAD     # dx without w_g
    assert router(by(ok), a[0], a[1], None, 4, None, a[3], a[4], a[5], need, None) == BAD
    assert router(by(ok), a[0] + 8, a[1], a[2], 4, None, a[3], a[4], a[5], need, None) == BAD
    assert router(by(ok), a[0], a[1], a[2], 4, a[6] + 8, a[3], a[4], a[5], need, None) == BAD
    assert router(by(ok), a[0], a[1], a[2], 4, None, a[3], a[4], a[5] + 4, need, None) == BAD
    assert router(by(ok), a[0], a[1], a[2], 4, None, a[3], a[4], a[5], need - 1, None) == hm.HMOE_ERR_WORKSPACE
    assert router(by(ok), a[0], a[1], a[2], 4, None, a[3], a[4], None, need, None) == hm.HMOE_ERR_WORKSPACE
    assert router(by(eight), a[0], a[1], a[2], 4, None, a[3], a[4], a[5], 1 << 30, None) == hm.HMOE_ERR_UNSUPPORTED


def test_router_gradient_refuses_a_batch_that_is_not_the_last_pass(hm):
    """Before anything reaches the library: no pass yet, another token count than the last pass and every captured one."""
    import torch
    layer = hm.MoELayer.__new__(hm.MoELayer)
    layer.cache, layer.desc, layer.dt, layer.max_tokens, layer.w_router = None, hm.make_desc(64, 64, 8, 2, 8, hm.HMOE_F32), torch.float32, 9, None
    x = torch.zeros(4, 64)
    for last, captured in ((None, set()), (3, set()), (9, {1, 5})):
        layer._pass_tokens, layer._captured_passes = last, captured
        with pytest.raises(AssertionError, match="last forward pass was of %s tokens, x has 4" % last):
            layer.router_gradient(x, x)
    layer._pass_tokens, layer._captured_passes = 9, {4}
    with pytest.raises(AssertionError) as e:     # (accepted: the next check speaks)
        layer.router_gradient(x, x[:3])
    assert "last forward pass" not in str(e.value)
