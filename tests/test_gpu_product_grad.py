"""The gradients of the experts' products against their definitions in 64 bits."""
import pytest
import torch

from paper_2605_10670_amd import layer

import grad_util as gr
import layer_util as lu

pytestmark = pytest.mark.gpu
TORCH_OF = gr.TORCH_OF


class Case:
    """counts: rows of each slot; `spare` rows behind the last, which are NaN."""

    def __init__(self, seed, counts, K, I, dtype="bf16", gate=False, spare=0):
        g = lu.gen(seed)
        self.counts, self.K, self.I, self.dtype, self.gate = counts, K, I, dtype, gate
        self.N, self.P, self.rows = I * (2 if gate else 1), len(counts), sum(counts) + spare
        self.routed = sum(counts)
        self.offset = torch.tensor([0] + list(counts)).cumsum(0).to(torch.int32)
        t = TORCH_OF[dtype]
        self.grad_y, self.x = lu.randn(g, self.rows, I).to(t), lu.randn(g, self.rows, K).to(t)
        self.sums = (2 * lu.randn(g, self.rows, self.N)).to(t) if gate else None
        self.w = (lu.randn(g, self.P, self.N, K) * K ** -0.5).to(t)
        for v in (self.grad_y, self.x, self.sums):
            if v is not None and spare:
                v[self.routed:] = float("nan")

    def handle(self, w_dtype="bf16", **kw):
        return layer.ExpertProductGrad(num_slots=self.P, in_features=self.K, out_features=self.I, max_rows=self.rows, dtype=self.dtype,
                                       grad_w_dtype=w_dtype, gate=self.gate, **kw)

    def run(self, handle, w_dtype="bf16", dense=False, old=None, wanted="xw", stream=None):
        dev = lambda t: None if t is None else t.cuda()
        new = lambda shape, t: torch.full(shape, gr.SENTINEL, device="cuda").to(t)
        t = TORCH_OF[self.dtype]
        out = dict(grad_sums=new((self.rows, self.N), t) if self.gate else None,
                   grad_x=new((self.rows, self.K), t) if "x" in wanted else None, grad_w=None)
        if "w" in wanted:
            out["grad_w"] = new((self.P, self.N, self.K), TORCH_OF[w_dtype]) if old is None else old.cuda()
        handle.run(dev(self.grad_y), self.rows, offset=None if dense else dev(self.offset), x=dev(self.x) if "w" in wanted else None,
                   w=dev(self.w) if "x" in wanted else None, sums=dev(self.sums), accumulate=old is not None, stream=stream, **out)
        torch.cuda.synchronize()
        return {k: v.cpu() for k, v in out.items() if v is not None}

    def check(self, out, old=None):
        n = self.routed
        offset = self.offset.tolist()
        g = self.grad_y[:n]
        for name in ("grad_sums", "grad_x"):
            if name in out:
                spare = out[name][n:]
                assert (spare.float() == torch.tensor(gr.SENTINEL).to(spare.dtype).float()).all(), name
        if self.gate:
            want, err = gr.gate_grad(g, self.sums[:n])
            gr.check("grad_sums", out["grad_sums"][:n], want, err)
            g = out["grad_sums"][:n]
        want = gr.product_grads(g, self.x[:n] if "grad_w" in out else None, self.w if "grad_x" in out else None, offset, old)
        if "grad_x" in out:
            gr.check("grad_x", out["grad_x"][:n], *want["grad_x"])
        if "grad_w" in out:
            gr.check("grad_w", out["grad_w"], *want["grad_w"])


COUNTS = [
    [1], [0, 1, 0], [3, 0, 5, 1, 0, 0, 7], [63, 64, 65], [1, 130, 2], [257, 0, 31], [300], [16, 17, 15, 0], [0, 0], [600, 8]]
SIZES = [(8, 8), (64, 64), (256, 256), (264, 136), (520, 72), (128, 1032)]


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("K,I", SIZES)
def test_bf16(counts, K, I):
    c = Case(sum(counts) + K, counts, K, I, spare=5)
    w_dtype = "f32" if I % 16 == 8 else "bf16"
    h = c.handle(w_dtype)
    out = c.run(h, w_dtype)
    c.check(out)
    for wanted in ("x", "w"):   # each alone gives the same bits
        alone = c.run(h, w_dtype, wanted=wanted)
        for k, v in alone.items():
            assert torch.equal(v.float().nan_to_num(), out[k].float().nan_to_num()), k
    h.destroy()


@pytest.mark.parametrize("counts", [[1], [3, 0, 5, 1], [33, 70, 31], [300, 2], [0, 0]], ids=str)
@pytest.mark.parametrize("K,I", [(4, 4), (8, 12), (256, 64), (260, 132), (72, 520)])
@pytest.mark.parametrize("w_dtype", ["f32", "bf16"])
def test_f32(counts, K, I, w_dtype):
    if K % 8 and w_dtype == "bf16":
        K += 4   # (rows of 16 bytes)
    c = Case(sum(counts) + K, counts, K, I, dtype="f32", spare=3)
    h = c.handle(w_dtype)
    c.check(c.run(h, w_dtype))
    h.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,K,I", [([2, 0, 40, 1], 264, 72), ([70, 130], 64, 256), ([1], 16, 8)])
def test_gate(dtype, counts, K, I):
    c = Case(K, counts, K, I, dtype=dtype, gate=True, spare=4)
    h = c.handle("f32")
    out = c.run(h, "f32")
    c.check(out)
    # the gate's alone, and in place of the sums
    assert torch.equal(c.run(h, wanted="")["grad_sums"], out["grad_sums"])
    sums = c.sums.cuda()
    h.run(c.grad_y.cuda(), c.rows, offset=c.offset.cuda(), sums=sums, grad_sums=sums)
    n = c.routed
    assert torch.equal(sums.cpu()[:n], out["grad_sums"][:n]) and sums[n:].isnan().all()
    h.destroy()


def test_gates_far_from_zero():
    a = torch.tensor([-200.0, -104.0, -90.0, -30.0, -1e-30, 0.0, 1e-30, 30.0, 90.0, 200.0, 3e38, -3e38, 2.0, -1.2785, 1.2785, -2.0])
    rows = a.numel()
    c = Case(1, [rows], 16, 8, dtype="f32", gate=True)
    c.sums = torch.cat([a[:, None].expand(rows, 8), c.sums[:, 8:]], dim=1).contiguous()
    h = c.handle("f32")
    out = c.run(h, wanted="")
    assert not out["grad_sums"].isnan().any()   # (a gradient of 1.2 times 3e38 is beyond fp32, and infinite as its rounding)
    want, err = gr.gate_grad(c.grad_y, c.sums)
    gr.check("grad_sums", out["grad_sums"], want, err)


@pytest.mark.parametrize("dtype,w_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("counts", [[5, 0, 2], [0, 200, 90]], ids=str)
def test_added_to_what_is_there(dtype, w_dtype, counts):
    c = Case(3, counts, 264, 72, dtype=dtype, spare=1)
    old = lu.randn(lu.gen(8), c.P, c.N, c.K).to(TORCH_OF[w_dtype])
    h = c.handle(w_dtype)
    out = c.run(h, w_dtype, old=old)
    c.check(out, old=old)
    for p, n in enumerate(counts):
        if n == 0:
            assert torch.equal(out["grad_w"][p], old[p])
    h.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 20, 64, 500])
def test_one_matrix(dtype, rows):
    c = Case(rows, [rows], 392, 264, dtype=dtype)
    h = c.handle("f32")
    c.check(c.run(h, "f32", dense=True))
    h.destroy()


def test_no_rows():
    c = Case(1, [0, 0], 64, 64)
    h = c.handle("f32")
    gw = torch.full((2, 64, 64), 3.0, device="cuda")
    none = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    h.run(none, 0, offset=off, x=none, grad_w=gw, accumulate=True)
    assert (gw == 3).all()
    h.run(none, 0, offset=off, x=none, w=c.w.cuda(), grad_x=none, grad_w=gw)
    assert (gw == 0).all()


def test_slots_apart_in_memory():
    """Weights and gradients that are parts of larger slots; what lies between them stays."""
    c = Case(4, [3, 0, 70], 64, 72)
    size = c.N * c.K
    store = torch.full((3, size + 64), 5.0).bfloat16()
    store[:, 32:32 + size] = c.w.view(3, -1)
    grads = torch.full((3, size + 128), 6.0, device="cuda")
    h = c.handle("f32", slot_stride=(size + 64) * 2, grad_stride=(size + 128) * 4)
    gx = torch.empty((c.rows, c.K), dtype=torch.bfloat16, device="cuda")
    store = store.cuda()
    h.run(c.grad_y.cuda(), c.rows, offset=c.offset.cuda(), x=c.x.cuda(), w=store.data_ptr() + 64, grad_x=gx,
          grad_w=grads.data_ptr() + 64 * 4)
    torch.cuda.synchronize()
    grads = grads.cpu()
    assert (grads[:, :64] == 6).all() and (grads[:, 64 + size:] == 6).all()
    c.check(dict(grad_x=gx.cpu(), grad_w=grads[:, 64:64 + size].reshape(3, c.N, c.K)))


def test_many_slots_and_offsets_out_of_range():
    counts = [(i * 7) % 4 for i in range(300)]
    c = Case(5, counts, 72, 64)
    h = c.handle("f32")
    c.check(c.run(h, "f32"))
    # offsets beyond the rows are taken as their end
    c = Case(6, [4, 6], 64, 64)
    c.offset = torch.tensor([-3, 4, 99], dtype=torch.int32)
    h = c.handle("f32")
    out = c.run(h, "f32")
    c.offset = torch.tensor([0, 4, 10], dtype=torch.int32)
    c.check(out)


def test_infinities_and_nans_stay_in_their_rows_and_slots():
    c = Case(7, [40, 30, 70], 264, 136)
    c.grad_y[41, 3] = float("nan")
    c.x[41, 5] = float("inf")
    h = c.handle("f32")
    out = c.run(h, "f32")
    assert (~out["grad_x"].float().isfinite()).any(dim=1).nonzero().flatten().tolist() == [41]
    bad = ~out["grad_w"].isfinite()
    assert bad[1].any() and not bad[0].any() and not bad[2].any()


@pytest.mark.parametrize("gate", [False, True])
def test_against_differences(gate):
    """The slope of a weighted sum of the product's results along one direction of x and of w, by the forward kernel in fp32."""
    counts, K, I = [3, 2], 32, 16
    c = Case(8, counts, K, I, dtype="f32", gate=gate)
    off = c.offset.cuda()
    forward = layer.ExpertProduct(num_slots=2, in_features=K, out_features=I, max_rows=c.rows, x_dtype="f32", y_dtype="f32", gate=gate)
    def loss(x, w):
        y = torch.empty((c.rows, I), device="cuda")
        forward.run(x.cuda(), w.cuda(), y, c.rows, offset=off)
        return float((y.cpu().double() * c.grad_y.double()).sum())
    if gate:
        both = layer.ExpertProduct(num_slots=2, in_features=K, out_features=2 * I, max_rows=c.rows, x_dtype="f32", y_dtype="f32")
        sums = torch.empty((c.rows, 2 * I), device="cuda")
        both.run(c.x.cuda(), c.w.cuda(), sums, c.rows, offset=off)
        c.sums = sums.cpu()
    out = c.run(c.handle("f32"), "f32")
    g = lu.gen(9)
    step = 2.0 ** -7
    for name, at, grad in (("x", c.x, out["grad_x"]), ("w", c.w, out["grad_w"])):
        way = lu.randn(g, *at.shape) * (0.1 if name == "x" else 0.02)
        ends = [loss(at + s * step * way, c.w) if name == "x" else loss(c.x, at + s * step * way) for s in (1, -1)]
        slope, want = (ends[0] - ends[1]) / (2 * step), float((grad.double() * way.double()).sum())
        # 80 results of about 3 terms each: roundings of 2^-20 of their size over the step, third derivatives times step^2 / 6
        assert abs(slope - want) < 80 * 4 * 2.0 ** -20 / step + 80 * step ** 2, name


@pytest.mark.parametrize("dtype,w_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("counts,K,I", [([1], 64, 4096), ([700], 264, 1032), ([2000, 0, 1500], 72, 64), ([3, 0, 1, 9, 0], 520, 2048)], ids=str)
def test_sums_in_parts(dtype, w_dtype, counts, K, I):
    """Few tiles of many terms: divided between workgroups."""
    c = Case(len(counts), counts, K, I, dtype=dtype, spare=2)
    h = c.handle(w_dtype)
    c.check(c.run(h, w_dtype))
    old = lu.randn(lu.gen(8), c.P, c.N, c.K).to(TORCH_OF[w_dtype])
    c.check(c.run(h, w_dtype, old=old, wanted="w"), old=old)
    h.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,K,I", [([2990, 3003, 1, 2816], 2056, 72), ([60] * 39 + [61], 2056, 72), ([3, 0, 17, 1] * 60, 1032, 136),
                                        ([10700], 1288, 72)], ids=["256", "64", "16", "one"])
def test_tiles_of_every_size(dtype, counts, K, I):
    """Enough tokens a slot, and slots, for tiles of 256, 64 and 16 tokens, several to a workgroup."""
    c = Case(sum(counts), counts, K, I, dtype=dtype)
    h = c.handle("bf16")
    c.check(c.run(h, wanted="x"))
    c.check(c.run(h, wanted="w"))
    h.destroy()


@pytest.mark.parametrize("dtype,w_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("counts,K,I", [([0, 1, 33, 70, 64, 96, 2] * 8, 520, 264), ([5, 0, 40] * 60, 264, 72), ([3000], 264, 520), ([31, 65, 0, 32], 1288, 136)],
                         ids=lambda v: f"{len(v)} slots" if isinstance(v, list) else str(v))
def test_weights_tiles_of_every_size(dtype, w_dtype, counts, K, I):
    """Many and few tiles of 256 and 64 weight rows, with ends in every direction; also added to what is there."""
    case = Case(K + I, counts, K, I, dtype)
    handle = case.handle(w_dtype)
    case.check(case.run(handle, w_dtype, wanted="w"))
    old = lu.randn(lu.gen(9), case.P, case.N, case.K).to(TORCH_OF[w_dtype])
    case.check(case.run(handle, w_dtype, wanted="w", old=old), old)
    handle.destroy()


@pytest.mark.parametrize("counts", [[40, 0, 300, 2], [2, 1, 0, 3], [900, 500, 0, 0]], ids=str)
def test_captured_and_replayed(counts):
    """One graph for all row counts: the offsets are read on the device."""
    c = Case(10, counts, 264, 72, gate=True)
    h, other = c.handle("f32"), c.handle("f32")
    dev = [t.cuda() for t in (c.grad_y, c.x, c.w, c.sums, c.offset)]
    gy, x, w, sums, off = dev
    new = lambda: dict(grad_sums=torch.zeros_like(sums), grad_x=torch.zeros_like(x), grad_w=torch.zeros((c.P, c.N, c.K), device="cuda"))
    out = new()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        h.run(gy, c.rows, offset=off, x=x, w=w, sums=sums, stream=stream, **out)
    g = lu.gen(12)
    for replay in range(4):
        cuts = torch.randint(0, c.rows + 1, (c.P - 1,), generator=g).sort().values
        off[1:-1] = cuts.to(torch.int32).cuda()
        gy.copy_(lu.randn(g, *gy.shape))
        want = new()
        other.run(gy, c.rows, offset=off, x=x, w=w, sums=sums, **want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], want[k]), k
