"""Operators of a mixture-of-experts layer beyond its forward pass in bfloat16, as a program of this library calls them:

  ffn     the grouped expert FFN in 8-bit integers: one scale per token and one per output channel, sums in 32-bit
          integers, the intermediate rows quantised again before the down projection
  back    the gradient of the tokens' way to the experts and back: of the weighted sum (to the experts' outputs and to
          the gate weights) and of the row gather (to the layer's input)
  gates   the gradient of the gates (softmax over the chosen logits) and of the router's product

`own` chooses between the library's kernels and the same formulas in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

# Layer shapes of this repository's workloads, and two generic ones.  `popular`: routing prefers low expert ids.
SHAPES = {
    "toy": dict(hidden=256, ffn=512, experts=8, top_k=2, popular=False),
    "small": dict(hidden=1024, ffn=640, experts=16, top_k=2, popular=False),
    "mixtral": dict(hidden=4096, ffn=14336, experts=8, top_k=2, popular=False),
    "dsv2lite": dict(hidden=2048, ffn=1408, experts=64, top_k=6, popular=True),
    "stress": dict(hidden=2048, ffn=1408, experts=64, top_k=6, popular=False),
}


def _case(op, shape, tokens, dtype="bf16", name=None):
    case = dict(op=op, tokens=tokens, dtype=dtype, **SHAPES[shape])
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one token of a decoding sequence, many small experts: latency and a short weight stream
        _case("ffn", "dsv2lite", 1, name="ffn_i8_decode1"),
        # eight sequences decoding, large experts: the weight stream is everything
        _case("ffn", "mixtral", 8, name="ffn_i8_decode8"),
        # a short prompt through a small layer: a few rows per expert
        _case("ffn", "small", 77, name="ffn_i8_prefill77"),
        # a prompt with skewed routing: one expert with hundreds of rows, dozens with a handful
        _case("ffn", "dsv2lite", 1003, name="ffn_i8_prefill1003"),
        # a prompt through large experts, compute and weight stream about even
        _case("ffn", "mixtral", 517, name="ffn_i8_prefill517"),
        # the largest prefill batch
        _case("ffn", "stress", 16384, name="ffn_i8_prefill16384"),
        # the gradient's smallest call: a check on a small model in fp32
        _case("back", "toy", 16, "f32", name="back_f32_16"),
        # a training batch of odd size, skewed routing
        _case("back", "dsv2lite", 1003, name="back_1003"),
        # the largest training batch
        _case("back", "stress", 16384, name="back_16384"),
        # the same three for the gates and the router
        _case("gates", "toy", 16, "f32", name="gates_f32_16"),
        _case("gates", "dsv2lite", 1003, name="gates_1003"),
        _case("gates", "stress", 16384, name="gates_16384"),
    ]


def draw(rng):
    def between(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    op = rng.choice(["ffn", "ffn", "back", "gates"])
    if op == "ffn":
        top_k = rng.randint(1, 8)
        while True:
            hidden, ffn = 128 * between(1, 32), 128 * between(1, 112)
            experts = rng.randint(top_k, 96)
            tokens = between(1, 16384)
            if experts * hidden * ffn <= 4 * 10 ** 8 and tokens * top_k * hidden * ffn <= 16384 * 6 * 2048 * 1408:
                break
        return dict(op=op, tokens=tokens, dtype="bf16", hidden=hidden, ffn=ffn, experts=experts, top_k=top_k,
                    popular=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    while True:
        hidden, top_k, tokens = 16 * between(2, 256), rng.randint(1, 12), between(1, 16384)
        if tokens * top_k * hidden * (2 if dtype == "f32" else 1) <= 16384 * 6 * 2048:
            break
    experts = rng.randint(top_k, 160)
    if op == "gates":
        tokens = max(1, min(tokens, 16384 * 64 * 2048 // ((2 if dtype == "f32" else 1) * experts * hidden)))
    return dict(op=op, tokens=tokens, dtype=dtype, hidden=hidden, ffn=128, experts=experts, top_k=top_k, popular=rng.random() < 0.5)


def _torch_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _bias(case):
    """What popular experts have on top of their N(0, 1) logits."""
    p = np.array([(e + 1) ** -1.1 if case["popular"] else 1.0 for e in range(case["experts"])])
    return np.log(case["experts"] * p / p.sum())


def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, device="cuda", generator=gen) * std


def _routing(case, gen):
    """The choice of the K largest of random logits, its weights, and the stable order of the assignments by expert."""
    T, E, K = case["tokens"], case["experts"], case["top_k"]
    logits = _normal(gen, T, E) + torch.tensor(_bias(case), dtype=torch.float32, device="cuda")
    top, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    idx = idx[:, :K].to(torch.int32).contiguous()
    weights = torch.softmax(top[:, :K], dim=1).contiguous()
    flat = idx.flatten().long()
    perm = torch.sort(flat, stable=True)[1].to(torch.int32)
    inv = torch.empty_like(perm)
    inv[perm.long()] = torch.arange(T * K, dtype=torch.int32, device="cuda")
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    return dict(idx=idx, weights=weights, perm=perm, inv=inv, offsets=offsets, counts=counts.tolist())


def _tokens(case, gen):
    """Activations normalised as a layer's input is."""
    x = _normal(gen, case["tokens"], case["hidden"])
    return (x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-5)).to(_torch_dtype(case))


def _expert_weights(case, seed):
    """bfloat16 weights of expert after expert: [3, F * H] gate, up, down."""
    gen = torch.Generator(device="cuda").manual_seed(2 * seed + 1)
    for _ in range(case["experts"]):
        yield _normal(gen, 3, case["ffn"] * case["hidden"], std=0.02).to(torch.bfloat16)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(2 * seed)
    T, H, E, K, dt = case["tokens"], case["hidden"], case["experts"], case["top_k"], _torch_dtype(case)
    state = dict(case=case, **_routing(case, gen))
    if case["op"] == "ffn":
        state["x"] = _tokens(case, gen)
    elif case["op"] == "back":
        state["dy"] = _normal(gen, T, H, std=0.01).to(dt)
        state["o"] = _normal(gen, T * K, H, std=0.5).to(dt)          # the experts' outputs, in sorted order
        state["dx_sorted"] = _normal(gen, T * K, H, std=0.01).to(dt)  # the gradient of the experts' inputs
    else:
        state["x"] = _tokens(case, gen)
        state["w_g"] = _normal(gen, E, H, std=H ** -0.5).to(dt)
        state["d_weights"] = _normal(gen, T, K, std=0.1)
        state["add"] = _normal(gen, T, H, std=0.01).to(dt)            # what has reached the input on other ways
    return state


def _quantise_rows(v):
    """fp32 rows -> (whole numbers in -127 .. 127, scale per row)."""
    amax = v.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100)
    return torch.round(v * 127.0 / amax), amax / 127.0


def prepare(case, seed):
    state = _inputs(case, seed)
    T, H, F, E, K = (case[k] for k in ("tokens", "hidden", "ffn", "experts", "top_k"))
    if case["op"] == "ffn" and not own:
        codes, scales = [], []
        for w in _expert_weights(case, seed):
            parts = [_quantise_rows(m.float()) for m in (w[0].view(F, H), w[1].view(F, H), w[2].view(H, F))]
            codes.append([q.to(torch.int8) for q, _ in parts])
            scales.append([s for _, s in parts])
        state.update(codes=codes, scales=scales)
    if own:
        import paper_2504_05897_amd as hm
        dtype = hm.HMOE_BF16_I8 if case["op"] == "ffn" else hm.HMOE_F32 if case["dtype"] == "f32" else hm.HMOE_BF16
        state.update(hm=hm, desc=hm.make_desc(H, F, E, K, E, dtype))
        dev, dt = "cuda", _torch_dtype(case)
        if case["op"] == "ffn":
            experts = []
            host = torch.empty(E, 3, F * H, dtype=torch.bfloat16, pin_memory=True)
            for e, w in enumerate(_expert_weights(case, seed)):
                host[e].copy_(w, non_blocking=True)
            torch.cuda.synchronize()
            for w in host.view(torch.int16).numpy().view(np.uint16):
                experts.append((w[0].reshape(F, H), w[1].reshape(F, H), w[2].reshape(H, F)))
            state["layer"] = hm.MoELayer(state["desc"], experts, max_tokens=1, host_copies=False)
            state["ws_bytes"] = hm.hmoe_ffn_workspace_bytes(state["desc"], T * K)
            state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device=dev)
            state["out"] = torch.empty(T * K, H, dtype=dt, device=dev)
        elif case["op"] == "back":
            state["do"] = torch.empty(T * K, H, dtype=dt, device=dev)
            state["dw"] = torch.empty(T, K, dtype=torch.float32, device=dev)
            state["dx"] = torch.empty(T, H, dtype=dt, device=dev)
        else:
            state["d_logits"] = torch.empty(T, E, dtype=torch.float32, device=dev)
            state["dx"] = torch.empty(T, H, dtype=dt, device=dev)
            state["dw_g"] = torch.empty(E, H, dtype=torch.float32, device=dev)
            state["ws_bytes"] = hm.hmoe_router_backward_workspace_bytes(state["desc"], T)
            state["ws"] = torch.empty(state["ws_bytes"], dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()
    return state


def _run_own(s):
    hm, desc, case = s["hm"], s["desc"], s["case"]
    T, A = case["tokens"], case["tokens"] * case["top_k"]
    if case["op"] == "ffn":
        hm.hmoe_expert_ffn_grouped_gather(desc, s["layer"].cache, s["x"], s["perm"], s["offsets"], A, None, s["out"], s["ws"],
                                          s["ws_bytes"])
        return s["out"]
    if case["op"] == "back":
        hm.hmoe_combine_backward(desc, s["dy"], s["o"], s["inv"], s["weights"], T, s["do"], s["dw"])
        hm.hmoe_permute_backward(desc, s["dx_sorted"], s["inv"], T, None, s["dx"])
        return [s["do"], s["dw"], s["dx"]]
    hm.hmoe_route_backward(desc, s["idx"], s["weights"], s["d_weights"], T, s["d_logits"])
    hm.hmoe_router_backward(desc, s["x"], s["w_g"], s["d_logits"], T, s["add"], s["dx"], s["dw_g"], s["ws"], s["ws_bytes"])
    return [s["d_logits"], s["dx"], s["dw_g"]]


def _plain_ffn(s):
    case = s["case"]
    out = torch.empty(case["tokens"] * case["top_k"], case["hidden"], dtype=torch.bfloat16, device="cuda")
    tokens = torch.div(s["perm"], case["top_k"], rounding_mode="floor").long()
    first = 0
    for (gate, up, down), (s_gate, s_up, s_down), n in zip(s["codes"], s["scales"], s["counts"]):
        if n == 0:
            continue
        q, s_x = _quantise_rows(s["x"][tokens[first:first + n]].float())
        g = (q @ gate.float().t()) * s_x * s_gate.t()
        u = (q @ up.float().t()) * s_x * s_up.t()
        q, s_h = _quantise_rows(g / (1.0 + torch.exp(-g)) * u)
        out[first:first + n] = ((q @ down.float().t()) * s_h * s_down.t()).to(torch.bfloat16)
        first += n
    return out


def _plain_back(s):
    case = s["case"]
    T, H, K = case["tokens"], case["hidden"], case["top_k"]
    rows = s["inv"].long()
    dy = s["dy"].float()
    do = torch.empty_like(s["o"])
    do[rows] = (s["weights"][:, :, None] * dy[:, None, :]).to(do.dtype).view(T * K, H)
    dw = (s["o"][rows].float().view(T, K, H) * dy[:, None, :]).sum(2)
    dx = s["dx_sorted"][rows].float().view(T, K, H).sum(1).to(do.dtype)
    return [do, dw, dx]


def _plain_gates(s):
    case = s["case"]
    w, dw = s["weights"], s["d_weights"]
    d_logits = torch.zeros(case["tokens"], case["experts"], device="cuda")
    d_logits.scatter_(1, s["idx"].long(), w * (dw - (w * dw).sum(1, keepdim=True)))
    dx = (d_logits @ s["w_g"].float() + s["add"].float()).to(s["add"].dtype)
    return [d_logits, dx, d_logits.t().contiguous() @ s["x"].float()]


def run(state):
    if own:
        return _run_own(state)
    return {"ffn": _plain_ffn, "back": _plain_back, "gates": _plain_gates}[state["case"]["op"]](state)


def exact(case, seed):
    """The same from the definitions, in 64 bits."""
    s = _inputs(case, seed)
    T, H, F, E, K = (case[k] for k in ("tokens", "hidden", "ffn", "experts", "top_k"))

    def steps_of(rows):
        """A row in units of 1/127 of its largest magnitude, to the nearest whole number, and that unit.  (The product with
        127 is exact and the quotient the only rounding: half a unit stays half a unit.)"""
        largest = torch.clamp(rows.double().abs().max(dim=1).values, min=2.0 ** -100)
        return torch.round(127 * rows.double() / largest[:, None]), largest / 127

    if case["op"] == "ffn":
        out = torch.zeros(T * K, H, dtype=torch.float64, device="cuda")
        token_of = s["perm"].long() // K
        ends = np.cumsum(s["counts"])
        for e, w in enumerate(_expert_weights(case, seed)):
            lo, hi = int(ends[e]) - s["counts"][e], int(ends[e])
            if lo == hi:
                continue
            wg, wu, wd = (steps_of(m.double()) for m in (w[0].view(F, H), w[1].view(F, H), w[2].view(H, F)))
            for at in range(lo, hi, 4096):
                rows = slice(at, min(at + 4096, hi))
                x, unit = steps_of(s["x"][token_of[rows]].double())
                gate = unit[:, None] * wg[1] * torch.matmul(x, wg[0].t())
                up = unit[:, None] * wu[1] * torch.matmul(x, wu[0].t())
                h, unit = steps_of(gate * torch.sigmoid(gate) * up)
                out[rows] = unit[:, None] * wd[1] * torch.matmul(h, wd[0].t())
        return out
    w = s["weights"].double()
    if case["op"] == "back":
        token_of = s["perm"].long() // K
        dy = s["dy"].double()
        do = torch.empty(T * K, H, dtype=torch.float64, device="cuda")
        dw = torch.empty(T * K, dtype=torch.float64, device="cuda")
        dx = torch.zeros(T, H, dtype=torch.float64, device="cuda")
        sorted_w = w.flatten()[s["perm"].long()]
        for at in range(0, T * K, 8192):  # in sorted order, a stretch of assignments at a time
            rows = slice(at, min(at + 8192, T * K))
            into = dy[token_of[rows]]
            do[rows] = sorted_w[rows, None] * into
            dw[s["perm"].long()[rows]] = (into * s["o"][rows].double()).sum(1)
        for j in range(K):
            dx += s["dx_sorted"][s["inv"].long().view(T, K)[:, j]].double()
        return [do, dw.view(T, K), dx]
    dw = s["d_weights"].double()
    # the Jacobian of softmax: d w_i / d l_j = w_i (delta_ij - w_j)
    jac = torch.diag_embed(w) - w[:, :, None] * w[:, None, :]
    chosen = (jac * dw[:, :, None]).sum(1)
    d_logits = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    for j in range(K):
        d_logits[torch.arange(T, device="cuda"), s["idx"][:, j].long()] += chosen[:, j]
    dx = torch.matmul(d_logits, s["w_g"].double()) + s["add"].double()
    return [d_logits, dx, torch.matmul(d_logits.t().contiguous(), s["x"].double())]


def work(case):
    T, H, F, E, K = (case[k] for k in ("tokens", "hidden", "ffn", "experts", "top_k"))
    A, elem = T * K, 4 if case["dtype"] == "f32" else 2
    if case["op"] == "ffn":
        # experts that a batch of this size touches on average (each one's weights are read once)
        rng, bias, batches = np.random.default_rng(0), _bias(case), 64 if T <= 256 else 4
        touched = 0.0
        for _ in range(batches):
            chosen = np.argpartition(-(rng.standard_normal((min(T, 4096), E)) + bias), K - 1, axis=1)[:, :K]
            touched += len(np.unique(chosen)) / batches
        weights = touched * (3 * H * F + 4 * (2 * F + H))
        return {"bytes": weights + 2 * T * H + 2 * A * H + 4 * (A + E + 1), "flops": 6.0 * H * F * A}
    if case["op"] == "back":
        return {"bytes": elem * H * (2 * T + 3 * A) + 8 * A + 8 * A, "flops": 4.0 * A * H}
    return {"bytes": elem * H * (3 * T + E) + 4 * E * H + 4 * T * E + 12 * A, "flops": 4.0 * T * E * H}
