"""64-bit statements of the layer's operators and the bounds of what fp32 sums may be off, for the GPU tests."""
import torch

GROUP = 128
TORCH_OF = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float32)


def quantise(v, rows):
    """fp32 [..., N, K] -> codes (float8) and a scale for each `rows` rows x 128 channels (a ragged last block allowed)."""
    n, k = v.shape[-2:]
    codes, scales = torch.empty(v.shape, dtype=torch.float8_e4m3fn), []
    for r in range(0, n, rows):
        b = v[..., r:r + rows, :]
        b = b.reshape(*b.shape[:-1], k // GROUP, GROUP)
        s = b.abs().amax(dim=(-3, -1)) / 448
        s = torch.where(s == 0, torch.ones_like(s), s)
        q = (b / s[..., None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        codes[..., r:r + rows, :] = q.reshape(*q.shape[:-2], k)
        scales.append(s)
    return codes, torch.stack(scales, dim=-2)


def dequantise(codes, scale, rows):
    n = codes.shape[-2]
    s = scale.double().repeat_interleave(rows, dim=-2)[..., :n, :].repeat_interleave(GROUP, dim=-1)
    return codes.double() * s


def e4m3_gap(q):
    """Half the distance between e4m3 neighbours around |q| <= 448 (rounded up at powers of two)."""
    _, e = torch.frexp(q.abs().clamp(min=2.0 ** -6, max=448.0))
    return torch.ldexp(torch.ones_like(q), e - 5)


def check_codes(code, scale, exact, err):
    """Codes and scales of `exact` (64 bits) known to `err` (absolute, elementwise)."""
    n, h = exact.shape
    groups = scale.shape[1]
    group = h // groups
    top = exact.abs().view(n, groups, group).amax(dim=2)
    err_top = err.view(n, groups, group).amax(dim=2)
    want = torch.where(top == 0, torch.ones_like(top), top / 448)
    assert ((scale.double() - want).abs() <= err_top / 448 + want * 2.0 ** -23 + 2.0 ** -149).all(), "scales"
    wide = scale.double().repeat_interleave(group, dim=1)
    q = exact / wide
    off = (code.double() - q.clamp(-448, 448)).abs()
    slack = err / wide + q.abs() * 2.0 ** -22
    assert (off <= e4m3_gap(q.abs() + slack) + slack).all(), "codes"


def check_rounded(y, exact, err):
    """y is the rounding of an fp32 value within `err` of `exact`: rounding keeps the order, so y lies between the
    roundings of both ends."""
    low, high = ((exact + s * err).float().to(y.dtype) for s in (-1, 1))
    bad = ~((low <= y) & (y <= high))
    off = ((y.double() - exact).abs() / err.clamp(min=1e-300))[bad]
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outputs off, worst {float(off.max()):.3g} of the bound"


def product_case(seed, counts, K, N, x="bf16", gate=False, spare=0):
    """Inputs on the CPU and the exact sums: rows of every slot in counts, `spare` rows behind the last."""
    g = gen(seed)
    P, rows = len(counts), sum(counts) + spare
    weight_rows = N * (2 if gate else 1)
    xf = randn(g, rows, K)
    wf = randn(g, P, weight_rows, K) * K ** -0.5
    c = dict(P=P, rows=rows, K=K, N=N, xt=x, gate=gate, x_scale=None, w_scale=None)
    c["offset"] = torch.tensor([0] + list(counts)).cumsum(0).to(torch.int32)
    if x == "fp8":
        c["x"], c["x_scale"] = quantise(xf, 1)
        c["w"], c["w_scale"] = quantise(wf, GROUP)
        xd, wd = dequantise(c["x"], c["x_scale"], 1), dequantise(c["w"], c["w_scale"], GROUP)
    else:
        c["x"], c["w"] = xf.to(TORCH_OF[x]), wf.to(TORCH_OF[x])
        xd, wd = c["x"].double(), c["w"].double()
    exact(c, xd, wd)
    return c


def exact(c, xd, wd):
    """c["sums"] in 64 bits, and c["sum_err"], what K additions in fp32 (in any order, each term and each sum rounded,
    or cut off by a matrix core's alignment) may be off: K * 2^-23 of the sum of magnitudes."""
    K = c["K"]
    s = torch.zeros((c["rows"], wd.shape[1]), dtype=torch.float64)
    m = torch.zeros_like(s)
    off = c["offset"].tolist()
    for p in range(c["P"]):
        lo, hi = off[p], off[p + 1]
        s[lo:hi] = xd[lo:hi] @ wd[p].t()
        m[lo:hi] = xd[lo:hi].abs() @ wd[p].abs().t()
    c["sums"], c["sum_err"] = s, m * (K + 8) * 2.0 ** -23
    c["xd"], c["wd"], c["routed"] = xd, wd, off[-1]


def lost_by_alignment(c):
    """What the matrix cores' 8-bit forms may lose: of every 8 neighbouring products each keeps the bits down to 2^-13 of
    the largest."""
    lost = torch.zeros_like(c["sums"])
    off = c["offset"].tolist()
    for p in range(c["P"]):
        x, w = c["xd"][off[p]:off[p + 1]].cuda().float(), c["wd"][p].cuda().float()
        if x.shape[0]:
            part = sum((x[:, None, k:k + 8] * w[None, :, k:k + 8]).abs().amax(dim=2).double() for k in range(0, c["K"], 8))
            lost[off[p]:off[p + 1]] = part.cpu() * 8 * 2.0 ** -13 * (1 + 2.0 ** -22)
    return lost


def result(c, y):
    """(the product in 64 bits, what it may be off before it is rounded to y)."""
    N, s, e = c["N"], c["sums"], c["sum_err"]
    if c["xt"] == "fp8" and y == "bf16":
        e = e + lost_by_alignment(c)
    if not c["gate"]:
        return s, e
    a, u = s[:, :N], s[:, N:]
    act = a * torch.sigmoid(a)
    # |silu'| < 1.1; the exponential, the quotient and the product round a few times each
    err = 1.1 * e[:, :N] * (u.abs() + e[:, N:]) + act.abs() * e[:, N:] + (act * u).abs() * 16 * 2.0 ** -23
    return act * u, err


SENTINEL = 77.0


def run_product(c, y="bf16", product=None, dense=False, stream=None):
    """The case through layer.ExpertProduct -> (y, y_scale) on the CPU; rows outside the slots start as SENTINEL."""
    from paper_2605_10670_amd import layer
    dev = lambda t: None if t is None else t.cuda()
    out = torch.full((c["rows"], c["N"]), SENTINEL, device="cuda").to(TORCH_OF[y])
    y_scale = torch.full((c["rows"], c["N"] // GROUP), SENTINEL, device="cuda") if y == "fp8" else None
    own = product is None
    if own:
        product = layer.ExpertProduct(num_slots=c["P"], in_features=c["K"], out_features=c["N"], x_dtype=c["xt"], y_dtype=y,
                                      gate=c["gate"], max_rows=c["rows"])
    product.run(dev(c["x"]), dev(c["w"]), out, c["rows"], offset=None if dense else dev(c["offset"]),
                x_scale=dev(c["x_scale"]), w_scale=dev(c["w_scale"]), y_scale=y_scale, stream=stream)
    torch.cuda.synchronize()
    if own:
        product.destroy()
    return out.cpu(), None if y_scale is None else y_scale.cpu()


def check_product(c, y, out, y_scale):
    n = c["routed"]
    assert (out[n:].float() == torch.tensor(SENTINEL).to(out.dtype).float()).all(), "rows outside the slots were written"
    want, err = (t[:n] for t in result(c, y))
    if y == "fp8":
        assert (y_scale[n:] == SENTINEL).all()
        check_codes(out[:n], y_scale[:n], want, err)
    else:
        check_rounded(out[:n], want, err + 2.0 ** -126)
