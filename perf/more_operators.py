"""The backward pass of an MoE layer, and the layer norm, as timed cases.

A case is one pass through one operator:

  kind "combine_grad"   grad_y[row_of[t, j]] = w[t, j] * grad_out[t], and the weights' gradients <grad_out[t], y[row_of[t, j]]>
  kind "dispatch_grad"  grad_x[t] = the sum of the gradients of the rows that token t was sent as
  kind "norm"           sum = x + residual and its layer norm (mean subtracted, bias)
  kind "norm_grad"      the gradients of a norm ("centred": the layer norm, else the root-mean-square norm): of its rows, its
                        gain and its bias
  kind "product_grad"   the gradients of the experts' products: of the rows ("x"), of every slot's weights ("w"), with the gate's
                        SiLU and product in between ("gate").  slots 0: no slots, all rows times one matrix
  kind "route_grad"     the gradient of the router's weights with respect to the logits

Sizes are those of this repository's workloads (7168 channels, 256 experts, top-8, 32 ranks of 8+1 slots; 4096 channels, 16
ranks; the ragged 2880 channels, top-6, 24 ranks of 4+1 slots), the experts' inner sizes 2048, 1408 and 1024.
"""
import functools
import math

import torch

own = False

TORCH_OF = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES_OF = {"f32": 4, "bf16": 2}
EPSILON = 1e-6


def _tokens(name, kind, tokens, hidden, topk, ranks, primary, **kw):
    return dict(dict(name=name, kind=kind, tokens=tokens, hidden=hidden, topk=topk, ranks=ranks, primary=primary, failed=0,
                     skew=0.0, y="bf16", out="bf16"), **kw)


def _norm(name, tokens, hidden, x="bf16", **kw):
    return dict(dict(name=name, kind="norm", tokens=tokens, hidden=hidden, x=x, y="bf16", residual=True, bias=True), **kw)


def _norm_grad(name, tokens, hidden, x="bf16", **kw):
    return dict(dict(name=name, kind="norm_grad", tokens=tokens, hidden=hidden, x=x, y="bf16", centred=False, stream=True), **kw)


def _product(name, tokens, topk, slots, inner, outer, **kw):
    """The product from rows of `inner` features to `outer` (gated: the two halves of 2 * outer)."""
    return dict(dict(name=name, kind="product_grad", tokens=tokens, topk=topk, slots=slots, empty=0, inner=inner, outer=outer,
                     x="bf16", w="bf16", gate=False, skew=0.0, dropped=0, wanted="xw"), **kw)


def _route(name, tokens, experts, topk, **kw):
    return dict(dict(name=name, kind="route_grad", tokens=tokens, experts=experts, topk=topk, x="f32", over_all=False, blocked=0,
                     skew=0.0), **kw)


def listed():
    return [
        # the smallest batch of a fine-tuned layer, one token a rank: latency counts
        _tokens("combine-grad-32", "combine_grad", 32, 7168, 8, 32, 8),
        # a ragged batch of the smaller model with a rank lost, fp32 residual stream
        _tokens("combine-grad-5976", "combine_grad", 5976, 2880, 6, 24, 4, failed=1, skew=0.3, out="f32"),
        # a full batch after two failures, hot experts
        _tokens("dispatch-grad-16384", "dispatch_grad", 16384, 7168, 8, 32, 8, failed=2, skew=0.6),
        # a ragged batch of the smaller model, fp32 residual stream: the forward layer norm
        _norm("layer-norm-5976", 5976, 2880, "f32"),
        # a few tokens: latency, and a gain's gradient out of few rows
        _norm_grad("layer-norm-grad-64", 64, 7168, centred=True),
        # a full batch of the norm in front of dispatch, with the gradient of the residual stream added
        _norm_grad("norm-grad-16384", 16384, 7168),
        # second product at few tokens: three or four rows a slot, all weights read and all their gradients written
        _product("down-grad-64", 64, 8, 144, 1024, 4096),
        # both factors of the first product of a ragged batch of the smaller model: sizes that are no multiples of a tile, fp32
        # gradients of the weights, slots of a failed rank empty, some pairs dropped
        _product("up-grad-5976", 5976, 6, 120, 2880, 2816, w="f32", empty=5, skew=0.3, dropped=7),
        # first product of a full batch after a failure: the matrix cores' case
        _product("up-grad-16384", 16384, 8, 144, 4096, 2048, gate=True, empty=9),
        # the second product of an expert that every token goes to
        _product("shared-grad-4096", 4096, 1, 0, 2048, 7168),
        # the router at the lowest concurrency
        _route("route-grad-32", 32, 256, 8),
        # a full batch, weights relative to all logits, bf16
        _route("route-grad-16384", 16384, 256, 8, x="bf16", over_all=True, blocked=16, skew=0.6),
    ]


# What a drawn pass may cost at most: the largest listed one's multiplications and weights.
MOST_FLOPS, MOST_WEIGHTS = 8.79e12, 2.42e9


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    while True:
        kind = rng.choices(["combine_grad", "dispatch_grad", "norm", "norm_grad", "product_grad", "route_grad"],
                           [15, 8, 8, 17, 42, 10])[0]
        if kind in ("combine_grad", "dispatch_grad"):
            ranks, primary = rng.choice([(32, 8), (16, 8), (24, 4), (4, 4), (1, 16)])
            hidden = rng.choice([7168, 4096, 2880, 8 * rng.randint(16, 1024)])
            c = _tokens("", kind, ranks * _log_uniform(rng, 1, 16384 // ranks), hidden, rng.choice([1, 2, 4, 6, 8, 8]), ranks,
                        primary, failed=rng.choice([0, 0, 1, 2]) if ranks > 2 else 0, skew=rng.choice([0.0, 0.3, 0.6]),
                        y=rng.choice(["bf16", "bf16", "f32"]), out=rng.choice(["bf16", "bf16", "f32"]))
        elif kind == "norm":
            c = _norm("", _log_uniform(rng, 1, 16384), 8 * rng.randint(16, 1024), rng.choice(["bf16", "bf16", "f32"]),
                      y=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.8, bias=rng.random() < 0.7)
        elif kind == "norm_grad":
            c = _norm_grad("", _log_uniform(rng, 1, 16384), 8 * rng.randint(16, 1024), rng.choice(["bf16", "bf16", "f32"]),
                           y=rng.choice(["bf16", "bf16", "f32"]), centred=rng.random() < 0.5, stream=rng.random() < 0.7)
        elif kind == "route_grad":
            experts = rng.choice([8, 16, 60, 64, 96, 128, 160, 256, 256, 384, 512])
            c = _route("", _log_uniform(rng, 1, 16384), experts, rng.choice([1, 2, 4, 6, 8, 8]), x=rng.choice(["f32", "bf16"]),
                       over_all=rng.random() < 0.4, blocked=rng.choice([0, 0, 1, experts // 8]), skew=rng.choice([0.0, 0.0, 0.6]))
        else:
            x = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
            inner, outer = (128 * rng.randint(4, 56) for _ in range(2))
            if rng.random() < 0.5:
                inner, outer = (8 * rng.randint(16, 400) for _ in range(2))
            slots = rng.choice([0, 0, 4, 9, 20, 40, 72, 120, 144])
            gate = rng.random() < 0.5
            # (with a gate in bf16, values next to a tie of grad_sums' rounding may fall either way: 1e-5 of grad_w, which bf16
            # covers and fp32 would show)
            w = "bf16" if gate and x == "bf16" else rng.choice(["bf16", "f32"])
            c = _product("", _log_uniform(rng, 1, 16384), min(rng.choice([1, 2, 4, 6, 8, 8]), max(1, slots // 2)), slots, inner, outer,
                         x=x, w=w, gate=gate, empty=rng.choice([0, 0, slots // 10]),
                         skew=rng.choice([0.0, 0.0, 0.3]), wanted=rng.choice(["xw", "xw", "x", "w"]))
            c["dropped"] = rng.choice([0, 0, min(5, c["tokens"] // 4)])
            if work(c)["flops"] > MOST_FLOPS * (0.05 if x == "f32" else 0.5):
                continue
            if max(slots, 1) * inner * outer * (2 if gate else 1) > MOST_WEIGHTS * (0.25 if x == "f32" else 1):
                continue
        del c["name"]
        return c


# ---- inputs ------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _placement(R, primary):
    """What each slot holds: a rank's own experts, and in one redundant slot the first expert of the rank half way round."""
    slots = []
    for r in range(R):
        slots += [r * primary + s for s in range(primary)]
        slots.append((r + R // 2) % R * primary)
    return slots


def _layout(c, topk_idx):
    """row_of [T, k] as the library's layout of these indices gives it (-1: no row): replica t mod n of the n live ones,
    primary ones first; rows by slot, then by token."""
    T, k, R, primary = c["tokens"], c["topk"], c["ranks"], c["primary"]
    S, E = primary + 1, R * primary
    held = _placement(R, primary)
    lists = [[] for _ in range(E)]
    for redundant in (False, True):
        for p, e in enumerate(held):
            if (p % S >= primary) == redundant and p // S >= c["failed"]:
                lists[e].append(p)
    most = max(map(len, lists))
    table = torch.tensor([v + [-1] * (most - len(v)) for v in lists], device="cuda")
    live = torch.tensor([len(v) for v in lists], device="cuda")
    idx = topk_idx.long()
    token = torch.arange(T, device="cuda")[:, None]
    slot = table[idx, token % live[idx].clamp(min=1)]
    routed = slot >= 0
    order = torch.argsort(torch.where(routed, slot, R * S).flatten(), stable=True)  # pairs of a slot stay by token
    row = torch.empty(T * k, dtype=torch.long, device="cuda")
    row[order] = torch.arange(T * k, device="cuda")
    return torch.where(routed, row.view(T, k), -1)


def _lost(c):
    """How many of the experts have no live slot."""
    held, S = _placement(c["ranks"], c["primary"]), c["primary"] + 1
    return c["ranks"] * c["primary"] - len({e for p, e in enumerate(held) if p // S >= c["failed"]})


def _prepare_tokens(c, g):
    T, H, k, R, primary = c["tokens"], c["hidden"], c["topk"], c["ranks"], c["primary"]
    E = R * primary
    popular = torch.randperm(E, generator=g, device="cuda")
    score = _randn(g, T, E) - c["skew"] * torch.log(1.0 + popular)
    top = score.topk(k, dim=1)
    s = dict(case=c, topk_idx=top.indices.to(torch.int32), topk_w=torch.softmax(top.values, dim=1))
    s["row_of"] = _layout(c, s["topk_idx"])
    y, out = TORCH_OF[c["y"]], TORCH_OF[c["out"]]
    rows = _randn(g, T * k, H).to(y)
    if c["kind"] == "combine_grad":
        s["y"] = rows
        s["grad_out"] = (_randn(g, T, H) * 1e-3).to(out)
        s["grad_y"] = torch.zeros((T * k, H), dtype=y, device="cuda")
        s["grad_w"] = torch.zeros((T, k), device="cuda")
    else:
        s["grad_recv"] = rows
        s["grad_x"] = torch.zeros((T, H), dtype=out, device="cuda")
    if own:
        from paper_2605_10670_amd import binding
        s["ctx"] = ctx = binding.Context(num_ranks=R, slots_per_rank=primary + 1, primary_slots=primary, num_logical=E,
                                         max_tokens=T, topk=k, hidden=H, x_dtype=c["y"], y_dtype=c["y"], out_dtype=c["out"],
                                         strict_coverage=False)
        ctx.update_placement(_placement(R, primary))
        ctx.set_membership([int(r >= c["failed"]) for r in range(R)])
        ctx.dispatch_layout(s["topk_idx"], T)
    return s


def _stream_rows(g, T, H, dtype):
    # a residual stream with a few large channels
    large = 1 + 8 * (torch.rand(H, generator=g, device="cuda") < 0.01)
    return (_randn(g, T, H) * large * 2 + 0.1).to(dtype)


def _prepare_norm(c, g):
    T, H, dt = c["tokens"], c["hidden"], TORCH_OF[c["x"]]
    return dict(case=c, x=_randn(g, T, H).to(dt), residual=_stream_rows(g, T, H, dt) if c["residual"] else None,
                gain=(1 + 0.2 * _randn(g, H)).to(torch.bfloat16),
                bias=(0.2 * _randn(g, H)).to(torch.bfloat16) if c["bias"] else None,
                sum=torch.empty((T, H), dtype=dt, device="cuda") if c["residual"] else None,
                y=torch.empty((T, H), dtype=TORCH_OF[c["y"]], device="cuda"))


def _prepare_norm_grad(c, g):
    T, H, dt = c["tokens"], c["hidden"], TORCH_OF[c["x"]]
    return dict(case=c, h=_stream_rows(g, T, H, dt), gain=(1 + 0.2 * _randn(g, H)).to(torch.bfloat16),
                grad_y=(_randn(g, T, H) * 1e-3).to(TORCH_OF[c["y"]]),
                grad_sum=(_randn(g, T, H) * 1e-3).to(dt) if c["stream"] else None,
                grad_h=torch.empty((T, H), dtype=dt, device="cuda"), grad_gain=torch.empty(H, device="cuda"),
                grad_bias=torch.empty(H, device="cuda") if c["centred"] else None)


def _prepare_product(c, g):
    T, k, P, K, I = c["tokens"], c["topk"], c["slots"], c["inner"], c["outer"]
    N = I * (2 if c["gate"] else 1)
    rows, dt = T * k, TORCH_OF[c["x"]]
    s = dict(case=c, rows=rows, offset=None, most=rows)
    if P:
        # rows of each slot as a router's choice among the live slots gives them
        live = P - c["empty"]
        score = _randn(g, T, live) - c["skew"] * torch.log(1.0 + torch.arange(live, device="cuda"))
        where = torch.randperm(P, generator=g, device="cuda")[:live]
        chosen = where[score.topk(k, dim=1).indices[:T - c["dropped"]]]
        count = torch.bincount(chosen.flatten(), minlength=P)
        s["offset"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).to(torch.int32)
        s["most"] = max(1, int(count.max()))
    elif c["dropped"]:
        s["rows"] = rows = rows - c["dropped"]
        s["most"] = rows
    s["grad_y"] = (_randn(g, rows, I) * 1e-3).to(dt)
    s["sums"] = _randn(g, rows, N).to(dt) if c["gate"] else None
    s["grad_sums"] = torch.zeros((rows, N), dtype=dt, device="cuda") if c["gate"] else None
    s["x"] = s["w"] = s["grad_x"] = s["grad_w"] = None
    if "w" in c["wanted"]:
        s["x"] = (_randn(g, rows, K) * (0.5 + torch.rand(K, generator=g, device="cuda"))).to(dt)
        s["grad_w"] = torch.zeros((max(P, 1), N, K), dtype=TORCH_OF[c["w"]], device="cuda")
    if "x" in c["wanted"]:
        s["w"] = torch.empty((max(P, 1), N, K), dtype=dt, device="cuda")
        for p in range(max(P, 1)):
            s["w"][p].normal_(0, K ** -0.5, generator=g)
        s["grad_x"] = torch.zeros((rows, K), dtype=dt, device="cuda")
    return s


def _prepare_route(c, g):
    T, E, k = c["tokens"], c["experts"], c["topk"]
    place = torch.randperm(E, generator=g, device="cuda")
    logits = _randn(g, T, E) - c["skew"] * torch.log(1.0 + place)
    logits[:, place[E - c["blocked"]:]] = -math.inf
    logits = logits.to(TORCH_OF[c["x"]])
    top = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    value, index = top.values[:, :k], top.indices[:, :k]
    chosen = value > -math.inf
    over = top.values if c["over_all"] else value
    w = torch.where(chosen, torch.exp(value - torch.logsumexp(over, dim=1, keepdim=True)), 0.0)
    return dict(case=c, logits=logits, topk_idx=torch.where(chosen, index, -1).to(torch.int32), topk_w=w,
                grad_w=_randn(g, T, k), grad_logits=torch.empty((T, E), dtype=logits.dtype, device="cuda"))


PREPARE = {"combine_grad": _prepare_tokens, "dispatch_grad": _prepare_tokens, "norm": _prepare_norm, "norm_grad": _prepare_norm_grad,
           "product_grad": _prepare_product, "route_grad": _prepare_route}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return PREPARE[case["kind"]](case, g)


# ---- the framework's operators -----------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _handle(kind, *shape):
    """What a program makes once for a layer's shape, as it makes its dispatch context."""
    from paper_2605_10670_amd import layer
    if kind == "norm":
        hidden, x, y = shape
        return layer.LayerNorm(hidden=hidden, in_dtype=x, gain_dtype="bf16", out_dtype=y, epsilon=EPSILON)
    if kind == "norm_grad":
        hidden, x, y, centred = shape
        return layer.NormGrad(hidden=hidden, in_dtype=x, gain_dtype="bf16", out_dtype=y, centred=centred, epsilon=EPSILON)
    if kind == "route_grad":
        experts, topk, x, over_all = shape
        return layer.Router(num_logical=experts, topk=topk, in_dtype=x, over_all=over_all)
    slots, inner, outer, x, w, gate, rows = shape
    return layer.ExpertProductGrad(num_slots=max(slots, 1), in_features=inner, out_features=outer, dtype=x, grad_w_dtype=w,
                                   gate=gate, max_rows=rows)


def _own_pass(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "combine_grad":
        s["ctx"].combine_grad(s["y"], s["topk_w"], s["grad_out"], s["grad_y"], s["grad_w"], c["tokens"])
        return dict(grad_y=s["grad_y"], grad_w=s["grad_w"])
    if kind == "dispatch_grad":
        s["ctx"].dispatch_grad(s["grad_recv"], s["grad_x"], c["tokens"])
        return dict(grad_x=s["grad_x"])
    if kind == "norm":
        _handle(kind, c["hidden"], c["x"], c["y"]).run(s["x"], s["gain"], c["tokens"], residual=s["residual"], bias=s["bias"],
                                                       sum=s["sum"], y=s["y"])
        return dict(sum=s["sum"], y=s["y"])
    if kind == "norm_grad":
        _handle(kind, c["hidden"], c["x"], c["y"], c["centred"]).run(
            s["h"], s["gain"], s["grad_y"], c["tokens"], grad_sum=s["grad_sum"], grad_h=s["grad_h"], grad_gain=s["grad_gain"],
            grad_bias=s["grad_bias"])
        return dict(grad_h=s["grad_h"], grad_gain=s["grad_gain"], grad_bias=s["grad_bias"])
    if kind == "route_grad":
        _handle(kind, c["experts"], c["topk"], c["x"], c["over_all"]).grad(
            s["topk_idx"], s["topk_w"], s["grad_w"], s["grad_logits"], c["tokens"], logits=s["logits"] if c["over_all"] else None)
        return dict(grad_logits=s["grad_logits"])
    _handle(kind, c["slots"], c["inner"], c["outer"], c["x"], c["w"], c["gate"], s["rows"]).run(
        s["grad_y"], s["rows"], offset=s["offset"], x=s["x"], w=s["w"], sums=s["sums"], grad_sums=s["grad_sums"],
        grad_x=s["grad_x"], grad_w=s["grad_w"])
    return dict(grad_sums=s["grad_sums"], grad_x=s["grad_x"], grad_w=s["grad_w"])


# ---- the plain forms ---------------------------------------------------------------------------
def _plain_combine_grad(s):
    c, row = s["case"], s["row_of"]
    routed = row >= 0
    grad_out = s["grad_out"].float()
    grad_y = torch.zeros((row.numel(), c["hidden"]), device=row.device)
    grad_y[row[routed]] = (grad_out[:, None, :] * s["topk_w"][:, :, None])[routed]
    each = (s["y"].float()[row.clamp(min=0)] * grad_out[:, None, :]).sum(dim=2)
    return dict(grad_y=grad_y.to(s["grad_y"].dtype), grad_w=torch.where(routed, each, 0.0))


def _plain_dispatch_grad(s):
    row = s["row_of"]
    each = s["grad_recv"].float()[row.clamp(min=0)]
    return dict(grad_x=torch.where((row >= 0)[:, :, None], each, 0.0).sum(dim=1).to(s["grad_x"].dtype))


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    d = h - h.mean(dim=1, keepdim=True)
    y = d * torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPSILON) * s["gain"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return dict(sum=h.to(s["x"].dtype) if s["residual"] is not None else None, y=y.to(s["y"].dtype))


def _plain_norm_grad(s):
    c, d, grad_y = s["case"], s["h"].float(), s["grad_y"].float()
    if c["centred"]:
        d = d - d.mean(dim=1, keepdim=True)
    inv = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPSILON)
    unit = d * inv
    v = grad_y * s["gain"].float()
    grad_h = v - unit * (v * unit).mean(dim=1, keepdim=True)
    if c["centred"]:
        grad_h = grad_h - v.mean(dim=1, keepdim=True)
    grad_h = grad_h * inv
    if s["grad_sum"] is not None:
        grad_h = grad_h + s["grad_sum"].float()
    return dict(grad_h=grad_h.to(s["h"].dtype), grad_gain=(grad_y * unit).sum(dim=0),
                grad_bias=grad_y.sum(dim=0) if c["centred"] else None)


def _plain_gate_grad(s):
    half = s["case"]["outer"]
    sums, grad_y = s["sums"].float(), s["grad_y"].float()
    gate, up = sums[:, :half], sums[:, half:]
    sigma = 1 / (1 + torch.exp(-gate))
    return torch.cat([grad_y * up * sigma * (1 + gate * (1 - sigma)), grad_y * gate * sigma], dim=1)


def _plain_product_grad(s):
    c, rows = s["case"], s["rows"]
    out = dict(grad_sums=None, grad_x=None, grad_w=None)
    grad = s["grad_y"].float()
    if s["offset"] is not None:
        # the slots' rows side by side, as many places as the fullest slot has
        offset = s["offset"].long()
        row = torch.arange(rows, device=grad.device)
        slot = torch.searchsorted(offset, row, right=True) - 1
        inside = slot < offset.numel() - 1
        slot = slot.clamp(max=offset.numel() - 2)
        at = (row - offset[slot]).clamp(max=s["most"] - 1)
        place = offset[:-1, None] + torch.arange(s["most"], device=grad.device)
        filled = (place < offset[1:, None])[:, :, None]
        place = place.clamp(max=rows - 1)
        side_by_side = lambda v: torch.where(filled, v[place], 0.0)
        back = lambda v: torch.where(inside[:, None], v[slot, at], 0.0)
    else:
        inside = torch.ones(rows, dtype=torch.bool, device=grad.device)
        side_by_side, back = (lambda v: v[None]), (lambda v: v[0])
    if c["gate"]:
        # (the products are those of the gradients as they are returned)
        rounded = torch.where(inside[:, None], _plain_gate_grad(s), 0.0).to(s["sums"].dtype)
        out["grad_sums"] = rounded
        grad = rounded.float()
    grad = side_by_side(grad)
    if s["grad_x"] is not None:
        out["grad_x"] = back(torch.bmm(grad, s["w"].float())).to(s["grad_x"].dtype)
    if s["grad_w"] is not None:
        x = side_by_side(s["x"].float())
        out["grad_w"] = torch.bmm(grad.transpose(1, 2).contiguous(), x).to(s["grad_w"].dtype)
    return out


def _plain_route_grad(s):
    c, w, grad_w = s["case"], s["topk_w"], s["grad_w"]
    idx = s["topk_idx"].long()
    chosen = idx >= 0
    inner = (w * grad_w).sum(dim=1, keepdim=True)
    grad = torch.zeros(s["logits"].shape, device=w.device)
    if c["over_all"]:
        logits = s["logits"].float()
        e = torch.exp(logits - logits.amax(dim=1, keepdim=True))
        grad = grad - e / e.sum(dim=1, keepdim=True) * inner
        each = w * grad_w
    else:
        each = w * (grad_w - inner)
    grad.scatter_add_(1, idx.clamp(min=0), torch.where(chosen, each, 0.0))
    return dict(grad_logits=grad.to(s["logits"].dtype))


PLAIN = {"combine_grad": _plain_combine_grad, "dispatch_grad": _plain_dispatch_grad, "norm": _plain_norm,
         "norm_grad": _plain_norm_grad, "product_grad": _plain_product_grad, "route_grad": _plain_route_grad}


def run(state):
    return _own_pass(state) if own else PLAIN[state["case"]["kind"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] in ("combine_grad", "dispatch_grad"):
        T, H, k = c["tokens"], c["hidden"], c["topk"]
        pairs = int(T * k * (1 - _lost(c) / (c["ranks"] * c["primary"])))
        token_bytes, row_bytes = H * BYTES_OF[c["out"]], H * BYTES_OF[c["y"]]
        if c["kind"] == "combine_grad":
            return {"bytes": T * token_bytes + 2 * pairs * row_bytes + 12 * T * k, "flops": 3 * pairs * H}
        return {"bytes": T * token_bytes + pairs * row_bytes + 4 * T * k, "flops": pairs * H}
    if c["kind"] == "norm":
        T, H = c["tokens"], c["hidden"]
        return {"bytes": T * H * (BYTES_OF[c["x"]] * (3 if c["residual"] else 1) + BYTES_OF[c["y"]]) + (4 if c["bias"] else 2) * H,
                "flops": 6 * T * H}
    if c["kind"] == "norm_grad":
        T, H = c["tokens"], c["hidden"]
        n = T * H * (BYTES_OF[c["x"]] * (3 if c["stream"] else 2) + BYTES_OF[c["y"]]) + 6 * H
        return {"bytes": n + (4 * H if c["centred"] else 0), "flops": 12 * T * H}
    if c["kind"] == "route_grad":
        T, E, k, b = c["tokens"], c["experts"], c["topk"], BYTES_OF[c["x"]]
        return {"bytes": T * (E * b * (2 if c["over_all"] else 1) + 12 * k), "flops": T * (3 * k + (4 * E if c["over_all"] else 0))}
    T, k, K, I, b = c["tokens"], c["topk"], c["inner"], c["outer"], BYTES_OF[c["x"]]
    N = I * (2 if c["gate"] else 1)
    rows, slots = (T - c["dropped"]) * k, max(c["slots"], 1)
    touched = 1.0
    if c["slots"]:  # slots that get a row at all
        live = c["slots"] - c["empty"]
        touched = live * (1 - (1 - k / live) ** (T - c["dropped"]))
    n, flops = rows * I * b * (5 if c["gate"] else 1), 0
    if "x" in c["wanted"]:
        n += touched * N * K * b + rows * K * b
        flops += 2 * rows * N * K
    if "w" in c["wanted"]:
        n += slots * N * K * BYTES_OF[c["w"]] + rows * K * b
        flops += 2 * rows * N * K
    return {"bytes": int(n), "flops": flops}


# ---- the definitions in 64 bits ----------------------------------------------------------------
def _exact_combine_grad(s):
    c = s["case"]
    g = s["grad_out"].double()
    grad_y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    grad_w = torch.zeros(s["topk_w"].shape, dtype=torch.float64, device="cuda")
    for j in range(c["topk"]):
        token = (s["row_of"][:, j] >= 0).nonzero().flatten()
        row = s["row_of"][token, j]
        grad_y[row] = s["topk_w"][token, j].double().unsqueeze(1) * g[token]
        grad_w[token, j] = torch.linalg.vecdot(s["y"][row].double(), g[token])
    return dict(grad_y=grad_y, grad_w=grad_w)


def _exact_dispatch_grad(s):
    grad = torch.zeros(s["grad_x"].shape, dtype=torch.float64, device="cuda")
    for j in range(s["case"]["topk"]):
        token = (s["row_of"][:, j] >= 0).nonzero().flatten()
        grad[token] += s["grad_recv"][s["row_of"][token, j]].double()
    return dict(grad_x=grad)


def _exact_norm(s):
    h = s["x"].double() if s["residual"] is None else s["x"].double() + s["residual"].double()
    var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
    y = s["gain"].double() * (h - mean) / (var + EPSILON).sqrt()
    if s["bias"] is not None:
        y += s["bias"].double()
    return dict(sum=h if s["residual"] is not None else None, y=y)


def _exact_norm_grad(s):
    centred = s["case"]["centred"]
    grad_h = torch.empty(s["h"].shape, dtype=torch.float64, device="cuda")
    H = s["h"].shape[1]
    grad_gain = torch.zeros(H, dtype=torch.float64, device="cuda")
    for at in range(0, s["h"].shape[0], 4096):
        part = slice(at, at + 4096)
        h, grad = s["h"][part].double(), s["grad_y"][part].double()
        d = h - h.sum(dim=1, keepdim=True) / H if centred else h
        root = (d.square().sum(dim=1, keepdim=True) / H + EPSILON).sqrt()
        v = grad * s["gain"].double()
        # d/dh of sum(v * d / root): v / root, less d times sum(v * d) / (H root^3), the mean taken out where d has none
        g = v / root - d * (v * d).sum(dim=1, keepdim=True) / (H * root ** 3)
        if centred:
            g -= g.sum(dim=1, keepdim=True) / H
        grad_h[part] = g
        grad_gain += (grad * d / root).sum(dim=0)
    if s["grad_sum"] is not None:
        grad_h += s["grad_sum"].double()
    return dict(grad_h=grad_h, grad_gain=grad_gain, grad_bias=s["grad_y"].double().sum(dim=0) if centred else None)


def _exact_product_grad(s):
    c, rows = s["case"], s["rows"]
    ends = [0, rows] if s["offset"] is None else s["offset"].tolist()
    out = dict(grad_sums=None, grad_x=None, grad_w=None)
    if c["gate"]:
        out["grad_sums"] = torch.zeros(s["sums"].shape, dtype=torch.float64, device="cuda")
    if s["grad_x"] is not None:
        out["grad_x"] = torch.zeros(s["grad_x"].shape, dtype=torch.float64, device="cuda")
    if s["grad_w"] is not None:
        out["grad_w"] = torch.zeros(s["grad_w"].shape, dtype=torch.float64, device="cuda")
    for p in range(len(ends) - 1):
        at = slice(ends[p], ends[p + 1])
        if ends[p] == ends[p + 1]:
            continue
        grad = s["grad_y"][at].double()
        if c["gate"]:
            a, b = s["sums"][at].double().split(c["outer"], dim=1)
            silu = torch.nn.functional.silu(a)
            slope = torch.sigmoid(a) + silu * torch.sigmoid(-a)
            out["grad_sums"][at] = torch.cat([grad * b * slope, grad * silu], dim=1)
            grad = out["grad_sums"][at].to(s["sums"].dtype).double()
        if s["grad_x"] is not None:
            out["grad_x"][at] = grad @ s["w"][p].double()
        if s["grad_w"] is not None:
            out["grad_w"][p] = grad.t().contiguous() @ s["x"][at].double()
    return out


def _exact_route_grad(s):
    c = s["case"]
    v = s["logits"].double()
    kept = torch.zeros(v.shape, dtype=torch.bool, device="cuda")
    grad_of = torch.zeros(v.shape, dtype=torch.float64, device="cuda")
    for j in range(c["topk"]):
        token = (s["topk_idx"][:, j] >= 0).nonzero().flatten()
        e = s["topk_idx"][token, j].long()
        kept[token, e] = True
        grad_of[token, e] = s["grad_w"][token, j].double()
    p = torch.softmax(v if c["over_all"] else v.masked_fill(~kept, -math.inf), dim=1)
    return dict(grad_logits=p * (grad_of - (p * grad_of).sum(dim=1, keepdim=True)))


EXACT = {"combine_grad": _exact_combine_grad, "dispatch_grad": _exact_dispatch_grad, "norm": _exact_norm,
         "norm_grad": _exact_norm_grad, "product_grad": _exact_product_grad, "route_grad": _exact_route_grad}


def exact(case, seed):
    s = prepare(case, seed)
    return EXACT[case["kind"]](s)
