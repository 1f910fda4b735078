"""Every kernel that the product's sizes may choose, at lengths of in_features that its pipeline treats apart, ragged slots and odd
widths, against the definition in 64 bits; which kernel ran is asserted."""
import pytest
import torch

import layer_util as lu
import product_util as pu

pytestmark = pytest.mark.gpu

CODES = [("fp8", "bf16", False), ("fp8", "f32", False), ("fp8", "bf16", True), ("fp8", "f32", True), ("fp8", "fp8", True)]
BF16 = [("bf16", "bf16", False), ("bf16", "f32", False), ("bf16", "bf16", True), ("bf16", "f32", True), ("bf16", "fp8", True)]
F32 = [("f32", "f32", False), ("f32", "bf16", False), ("f32", "f32", True), ("f32", "fp8", True)]
STEP = {"fp8": 128, "bf16": 64, "f32": 32}                          # channels
TAIL = {"fp8": 0, "bf16": 24, "f32": 12}                            # of a row that ends within a step


def make(seed, counts, K, N, x, gate):
    """Operands on the GPU, their exact values, rows of each slot by counts, two rows behind the last."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    P, rows, weight_rows = len(counts), sum(counts) + 2, N * (2 if gate else 1)
    xs, ws = randn(rows, K), randn(P, weight_rows, K) * K ** -0.5
    c = dict(offset=torch.tensor([0, *counts]).cumsum(0).to(torch.int32), K=K, N=N, gate=gate, routed=sum(counts), scales={})
    if x == "fp8":
        # (not normalised: every block has its own scale, and codes of every size)
        c["x"], c["w"] = (100 * xs).clamp(-448, 448).to(torch.float8_e4m3fn), (100 * K ** 0.5 * ws).clamp(-448, 448).to(torch.float8_e4m3fn)
        x_scale = (0.5 + torch.rand((rows, K // 128), generator=g, device="cuda")) / 100
        w_scale = (0.5 + torch.rand((P, -(-weight_rows // 128), K // 128), generator=g, device="cuda")) / 100 * K ** -0.5
        c["scales"] = dict(x_scale=x_scale, w_scale=w_scale)
        wide = lambda v, s, n: v.double() * s.double().repeat_interleave(n, dim=-2)[..., :v.shape[-2], :].repeat_interleave(128, dim=-1)
        c["xd"], c["wd"] = wide(c["x"], x_scale, 1), wide(c["w"], w_scale, 128)
    else:
        c["x"], c["w"] = xs.to(pu.TORCH_OF[x]), ws.to(pu.TORCH_OF[x])
        c["xd"], c["wd"] = c["x"].double(), c["w"].double()
    return c


def exact(c):
    """(the product in 64 bits, what it may be off before its last rounding): K additions of fp32 in any order."""
    sums = torch.zeros((c["routed"], c["wd"].shape[1]), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(sums)
    ends = c["offset"].tolist()
    for p in range(len(ends) - 1):
        if ends[p] < ends[p + 1]:
            a, b = c["xd"][ends[p]:ends[p + 1]], c["wd"][p].t().contiguous()
            sums[ends[p]:ends[p + 1]] = a @ b
            size[ends[p]:ends[p + 1]] = a.abs() @ b.abs()
    err = size * (c["K"] + 8) * 2.0 ** -23
    if not c["gate"]:
        return sums, err
    a, u, ea, eu = sums[:, :c["N"]], sums[:, c["N"]:], err[:, :c["N"]], err[:, c["N"]:]
    act = a * torch.sigmoid(a)
    return act * u, 1.1 * ea * (u.abs() + eu) + act.abs() * eu + (act * u).abs() * 16 * 2.0 ** -23


def check(form, seed, counts, K, N, x, y, gate, dense=False):
    c = make(seed, counts, K, N, x, gate)
    offset = None if dense else c["offset"].cuda()
    if dense:
        c["x"], n = c["x"][:c["routed"]], c["routed"]
        if x == "fp8":
            c["scales"]["x_scale"] = c["scales"]["x_scale"][:n].contiguous()
    out, y_scale, got = pu.run(c["x"], c["w"], offset, y, gate, xt=x, **c["scales"])
    assert got == form
    n = c["routed"]
    assert (out[n:].float() == torch.tensor(77.0).to(out.dtype).float()).all(), "rows outside the slots were written"
    want, err = exact(c)
    # besides the bound of every sum: errors in no common direction, of sqrt(K) * 2^-24 together (through the gate 2.2 times that and a few
    # roundings), and a bf16 result's 2^-9 each in the mean of squares at most
    together = ((2.2 * K ** 0.5 + 8) if gate else K ** 0.5) * 2.0 ** -24
    off = lambda a, b: float((a.double() - b).norm() / b.norm())
    if y == "fp8":
        assert (y_scale[n:] == 77.0).all()
        lu.check_codes(out[:n].cpu(), y_scale[:n].cpu(), want.cpu(), err.cpu())
        assert off(y_scale[:n], want.view(n, -1, 128).abs().amax(dim=2) / 448) <= together + 2.0 ** -24
    else:
        lu.check_rounded(out[:n], want, err + 2.0 ** -126)
        assert off(out[:n], want) <= together + (2.0 ** -8 if y == "bf16" else 0)


def odd(N, x, y, gate):
    """A width that is no multiple of a tile, where there may be one; codes with their weights' blocks are whole."""
    return N if y == "fp8" or (x == "fp8" and gate) else N - 56


# ---- a row or so a slot, the weights from memory to registers ---------------
@pytest.mark.parametrize("steps", list(range(1, 18)))
@pytest.mark.parametrize("x,y,gate", CODES + BF16 + F32)
def test_thin(x, y, gate, steps):
    """Steps around the number of those under way (three or four), with and without a tail; slots of no row, one, and more than a tile."""
    counts = [1] * 280 + [0] * 20 + [3, 0, 17, 0, 0, 0] + [1] * 30 + [0] * 30
    check("thin", steps, counts, steps * STEP[x] + TAIL[x] * (steps % 2), odd(128, x, y, gate), x, y, gate)


# ---- few rows ---------------------------------------------------------------
# (form, rows of the slots, out_features, those with the gate, with it where the results are codes)
FEW = [("few 1 1", (2, 0, 1), 456, 248, 256), ("few 2 1", (15,), 8200, 4104, 4224), ("few 2 1", (2, 0, 5), 2760, 1384, 1408),
       ("few 8 1", (16,), 16392, 8200, 8320), ("few 1 2", (30,), 456, 248, 256), ("few 4 2", (17,), 8200, 4104, 4224),
       ("few 1 4", (60,), 456, 248, 256), ("few 2 4", (33,), 4104, 2056, 2176)]


@pytest.mark.parametrize("form,counts,N,gated,codes", FEW)
@pytest.mark.parametrize("x,y,gate", CODES + BF16 + F32)
@pytest.mark.parametrize("steps", [2, 19])
def test_few(form, counts, N, gated, codes, x, y, gate, steps):
    """Fewer steps than wavefronts, and some two a wavefront, the last one's with a tail."""
    N = codes if y == "fp8" else gated if gate else N
    if x == "fp8" and gate:
        N = -(-N // 128) * 128
    check(form, steps, counts, steps * STEP[x] + TAIL[x], N, x, y, gate, dense=len(counts) == 1)


# ---- tiles ------------------------------------------------------------------
STEPS = [3, 4, 5, 6, 9]


@pytest.mark.parametrize("steps", STEPS)
@pytest.mark.parametrize("x,y,gate", CODES + BF16 + F32)
def test_tiles_of_64(x, y, gate, steps):
    """More of them than CUs, so that a workgroup goes on to a second one, of another slot."""
    counts = [0, 65, 1, 30] + [20 + 7 * (p % 9) for p in range(80)] + [0, 0, 64, 128, 3]
    check("tiled 1", steps, counts, steps * STEP[x] - TAIL[x], odd(512 if gate else 1024, x, y, gate), x, y, gate)


@pytest.mark.parametrize("steps", STEPS)
@pytest.mark.parametrize("x,y,gate", CODES + BF16 + F32)
def test_tiles_of_128(x, y, gate, steps):
    counts = [129, 0, 1, 128, 127] + [100 + p % 29 for p in range(112)] + [250, 0]
    check("tiled 2", steps, counts, steps * STEP[x] - TAIL[x], odd(384 if gate else 768, x, y, gate), x, y, gate)


@pytest.mark.parametrize("steps", STEPS)
@pytest.mark.parametrize("x,y,gate", BF16 + F32)
def test_tiles_of_256(x, y, gate, steps):
    counts = [257, 0, 256, 1, 255] + [240 + p % 50 for p in range(100)] + [700, 0, 17]
    check("tiled 4", steps, counts, steps * STEP[x] - TAIL[x], odd(384 if gate else 768, x, y, gate), x, y, gate)


@pytest.mark.parametrize("form,rows", [("tiled 2", 8190), ("tiled 4", 16381)])
@pytest.mark.parametrize("x,y,gate", CODES + BF16[:2])
def test_one_matrix(form, rows, x, y, gate):
    """All rows through one matrix, tiles of every CU side by side, then a second round of them."""
    if x == "fp8" and form == "tiled 4":
        form = "tiled 2"                                        # (the largest for codes)
    check(form, 1, (rows,), 7 * STEP[x] - TAIL[x], odd(512 if gate else 1024, x, y, gate), x, y, gate, dense=True)
