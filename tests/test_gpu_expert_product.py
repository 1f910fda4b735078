"""The experts' product against its definition in 64 bits: types, gates, ragged and empty slots, odd sizes, tails of
rows that are no whole step, strided weight stores, values that may not leak from one slot or row into another."""
import numpy as np
import pytest
import torch

import layer_util as lu

pytestmark = pytest.mark.gpu


def case_and_check(seed, counts, K, N, x, y, gate, spare=0, dense=False):
    c = lu.product_case(seed, counts, K, N, x, gate, spare)
    out, y_scale = lu.run_product(c, y, dense=dense)
    lu.check_product(c, y, out, y_scale)


COUNTS = {
    "one row": (1,), "one of many": (0, 0, 0, 1, 0), "none": (0, 0, 0), "empty ends": (0, 5, 0, 0, 17, 0),
    "edges": (15, 16, 17, 1, 31, 32, 33), "tiles": (63, 64, 65, 127, 128, 129, 0, 2), "skewed": (300, 1, 0, 2, 1, 0, 0, 3),
}


@pytest.mark.parametrize("counts", list(COUNTS))
@pytest.mark.parametrize("x,y,gate", [("bf16", "bf16", False), ("bf16", "f32", True), ("f32", "f32", False), ("f32", "bf16", True),
                                      ("fp8", "bf16", False), ("fp8", "f32", True), ("fp8", "fp8", True), ("bf16", "fp8", True),
                                      ("f32", "fp8", True)])
def test_slots_of_every_size(counts, x, y, gate):
    case_and_check(1, COUNTS[counts], 256, 256, x, y, gate, spare=3)


@pytest.mark.parametrize("K,N", [(8, 8), (16, 24), (64, 8), (72, 136), (120, 264), (128, 16), (136, 40), (1000, 8), (1408, 200), (192, 1000)])
@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("counts", [(3, 0, 18), (70, 150, 1)])
def test_sizes_that_are_no_multiples(K, N, x, y, gate, counts):
    case_and_check(2, counts, K, N, x, y, gate)


def test_rows_of_four_floats():
    case_and_check(3, (2, 20), 4, 4, "f32", "f32", False)
    case_and_check(3, (2, 200), 12, 20, "f32", "f32", True)


@pytest.mark.parametrize("K", [128, 256, 384, 640, 896, 1152, 2048])
@pytest.mark.parametrize("N,gate,y", [(8, False, "bf16"), (136, False, "f32"), (392, False, "bf16"), (128, True, "fp8"), (384, True, "bf16")])
@pytest.mark.parametrize("counts", [(5, 0, 40), (1, 130, 257)])
def test_scale_blocks(K, N, gate, y, counts):
    case_and_check(4, counts, K, N, "fp8", y, gate)


@pytest.mark.parametrize("rows", [1, 2, 7, 16, 17, 33, 64, 100, 129, 255, 300, 520])
@pytest.mark.parametrize("x,y,gate", [("fp8", "fp8", True), ("bf16", "bf16", False), ("fp8", "bf16", False), ("bf16", "f32", True),
                                      ("f32", "f32", False)])
def test_without_slots(rows, x, y, gate):
    case_and_check(5, (rows,), 512, 384, x, y, gate, dense=True)


@pytest.mark.parametrize("K,N", [(4096, 128), (7168, 256)])
@pytest.mark.parametrize("x,y,gate", [("fp8", "fp8", True), ("bf16", "bf16", False)])
@pytest.mark.parametrize("rows", [1, 5, 40, 200])
def test_long_rows(K, N, x, y, gate, rows):
    case_and_check(6, (rows,), K, N, x, y, gate, dense=True)


def test_many_slots():
    """More slots than a wavefront has lanes, most of them empty, tiles found across runs of empty ones."""
    rng = np.random.default_rng(7)
    for P in (63, 64, 65, 288, 1000):
        counts = rng.integers(0, 3, P) * (rng.random(P) < 0.4)
        counts[int(rng.integers(0, P))] = 45
        case_and_check(7, tuple(int(v) for v in counts), 64, 16, "bf16", "bf16", False, spare=2)


def test_no_rows_and_no_slots_with_rows():
    from paper_2605_10670_amd import layer
    p = layer.ExpertProduct(num_slots=2, in_features=64, out_features=64, max_rows=8)
    p.run(None, None, None, 0)
    w = torch.zeros((2, 64, 64), dtype=torch.bfloat16, device="cuda")
    x = torch.ones((8, 64), dtype=torch.bfloat16, device="cuda")
    y = torch.full((8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    p.run(x, w, y, 8, offset=torch.zeros(3, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert (y == 3).all()
    p.destroy()


@pytest.mark.parametrize("counts", [(4, 0, 33), (140, 2, 300)])
@pytest.mark.parametrize("x,gate", [("bf16", False), ("fp8", True)])
def test_weights_in_a_slot_major_store(counts, x, gate):
    """Weights and scales side by side in one store, as a repair moves them: strides, and a start within the slot."""
    from paper_2605_10670_amd import layer
    c = lu.product_case(8, counts, 256, 128, x, gate)
    P = c["P"]
    wb = c["w"].reshape(P, -1).view(torch.uint8)
    sb = c["w_scale"].reshape(P, -1).view(torch.uint8) if x == "fp8" else torch.empty((P, 0), dtype=torch.uint8)
    lead, gap = 64, 80
    stride = lead + wb.shape[1] + gap + (sb.shape[1] + 15) // 16 * 16
    store = torch.full((P, stride), 0x7f, dtype=torch.uint8)        # NaN codes where nothing belongs
    store[:, lead:lead + wb.shape[1]] = wb
    at = lead + wb.shape[1] + gap
    store[:, at:at + sb.shape[1]] = sb
    store = store.cuda()
    p = layer.ExpertProduct(num_slots=P, in_features=256, out_features=128, x_dtype=x, y_dtype="f32", gate=gate,
                            max_rows=c["rows"], slot_stride=stride, scale_stride=stride if x == "fp8" else None)
    y = torch.empty((c["rows"], 128), device="cuda")
    p.run(c["x"].cuda(), store.data_ptr() + lead, y, c["rows"], offset=c["offset"].cuda(),
          x_scale=None if x != "fp8" else c["x_scale"].cuda(), w_scale=None if x != "fp8" else store.data_ptr() + at)
    torch.cuda.synchronize()
    lu.check_product(c, "f32", y.cpu(), None)
    p.destroy()


@pytest.mark.parametrize("x,y,gate", [("bf16", "f32", False), ("fp8", "f32", True), ("f32", "f32", False)])
@pytest.mark.parametrize("counts", [(5, 20, 9), (130, 70, 140)])
@pytest.mark.parametrize("K", [128, 200])
def test_nan_and_infinity_stay_in_their_row_and_slot(x, y, gate, counts, K):
    if x == "fp8" and K % 128:
        K = 384
    c = lu.product_case(9, counts, K, 256, x, gate)
    clean, _ = lu.run_product(c, y)
    bad_row, bad_slot = counts[0] + 2, 2
    c["x"][bad_row, K - 1] = float("nan")
    c["w"][bad_slot, 3, 0] = float("nan")
    out, _ = lu.run_product(c, y)
    lo = counts[0] + counts[1]
    keep = torch.ones(c["rows"], dtype=torch.bool)
    keep[bad_row] = False
    keep[lo:] = False
    assert torch.equal(out[keep], clean[keep])
    assert out[bad_row].isnan().all()
    assert out[lo:, 3].isnan().all()
    others = torch.arange(256) != 3
    assert torch.equal(out[lo:, others], clean[lo:, others])


def test_all_zero_blocks():
    """A group of zeros has scale 1 and codes 0."""
    c = lu.product_case(10, (3, 30), 256, 256, "fp8", True)
    c["w"] = c["w"].float().index_fill(1, torch.arange(0, 128), 0.0).to(torch.float8_e4m3fn)
    lu.exact(c, lu.dequantise(c["x"], c["x_scale"], 1), lu.dequantise(c["w"], c["w_scale"], 128))
    out, y_scale = lu.run_product(c, "fp8")
    lu.check_product(c, "fp8", out, y_scale)
    assert (out[:, :128].float() == 0).all() and (y_scale[:, 0] == 1).all()


def test_captured_with_offsets_that_change():
    """One graph, replayed over other row counts: the grid does not depend on them."""
    from paper_2605_10670_amd import layer
    cases = [lu.product_case(11 + i, n, 256, 256, "bf16", False, spare=s)
             for i, (n, s) in enumerate([((40, 0, 25), 0), ((0, 65, 0), 0), ((1, 1, 1), 62), ((0, 0, 65), 0)])]
    p = layer.ExpertProduct(num_slots=3, in_features=256, out_features=256, y_dtype="f32", max_rows=65)
    x, w, off = (torch.empty_like(cases[0][k], device="cuda") for k in ("x", "w", "offset"))
    y = torch.empty((65, 256), device="cuda")
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        p.run(x, w, y, 65, offset=off, stream=side)
    for c in cases + cases[::-1]:
        for dst, k in ((x, "x"), (w, "w"), (off, "offset")):
            dst.copy_(c[k])
        y.fill_(lu.SENTINEL)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        lu.check_product(c, "f32", y.cpu(), None)
    p.destroy()


@pytest.mark.parametrize("K", [512, 1024, 1080, 2168, 7168])
@pytest.mark.parametrize("x,y,gate", [("fp8", "fp8", True), ("fp8", "f32", False), ("bf16", "bf16", True), ("f32", "f32", False)])
@pytest.mark.parametrize("counts", [(1,), (0, 3, 0, 16), (2, 1, 17, 0, 1)])
def test_few_rows_divide_in_features(K, x, y, gate, counts):
    """Few workgroups' worth of rows: parts of in_features by several workgroups, steps that do not divide evenly, a tail."""
    if x == "fp8":
        K = K // 128 * 128
    case_and_check(21, counts, K, 256, x, y, gate, spare=1)


def test_divided_product_twice_with_one_handle():
    """The words that count the parts are as they were after every call, also where a call has fewer tiles than the one before."""
    from paper_2605_10670_amd import layer
    p = layer.ExpertProduct(num_slots=4, in_features=1024, out_features=256, x_dtype="fp8", y_dtype="fp8", gate=True, max_rows=40)
    for i, counts in enumerate([(1, 0, 0, 0), (3, 1, 1, 3), (0, 0, 0, 0), (0, 16, 0, 17), (0, 0, 0, 2)] * 3):
        c = lu.product_case(22 + i, counts, 1024, 256, "fp8", True, spare=1)
        out, y_scale = lu.run_product(c, "fp8", product=p)
        lu.check_product(c, "fp8", out, y_scale)
    p.destroy()


def test_results_do_not_depend_on_the_run():
    c = lu.product_case(20, (1, 40, 300), 1024, 256, "fp8", True)
    first = lu.run_product(c, "fp8")
    for _ in range(3):
        again = lu.run_product(c, "fp8")
        assert torch.equal(first[0].view(torch.uint8), again[0].view(torch.uint8)) and torch.equal(first[1], again[1])


def test_refusals_of_a_call():
    """Addresses that are never read: every one of these returns before anything is queued."""
    from paper_2605_10670_amd import binding, layer
    A = 1 << 20
    bf16 = layer.ExpertProduct(num_slots=4, in_features=256, out_features=128, max_rows=16)
    fp8 = layer.ExpertProduct(num_slots=4, in_features=256, out_features=128, max_rows=16, x_dtype="fp8", y_dtype="fp8", gate=True)
    one = dict(x=A, w=A, y=A, rows=16, offset=A)
    whole = dict(one, x_scale=A, w_scale=A, y_scale=A)
    for p, good, bad in [(bf16, one, dict(rows=17)), (bf16, one, dict(rows=-1)), (bf16, one, dict(x=None)), (bf16, one, dict(w=None)),
                         (bf16, one, dict(y=None)), (bf16, one, dict(offset=None)), (bf16, one, dict(x_scale=A)),
                         (bf16, one, dict(w_scale=A)), (bf16, one, dict(y_scale=A)), (fp8, whole, dict(x_scale=None)),
                         (fp8, whole, dict(w_scale=None)), (fp8, whole, dict(y_scale=None))]:
        with pytest.raises(binding.EepError) as e:
            p.run(**{**good, **bad})
        assert e.value.code == binding.ERR_INVALID_ARG
    for name in ("x", "w", "y", "offset", "x_scale", "w_scale", "y_scale"):
        with pytest.raises(binding.EepError) as e:
            fp8.run(**{**whole, name: A + 2})
        assert e.value.code == binding.ERR_ALIGN
    with pytest.raises(ValueError):
        bf16.run(**{**one, "x": torch.zeros((15, 256), dtype=torch.bfloat16, device="cuda")})
    bf16.destroy()
    fp8.destroy()


@pytest.mark.parametrize("rows,K,N,y", [(70000, 32768, 128, "f32"), (70000, 64, 16384, "f32")])
def test_arrays_past_four_gigabytes(rows, K, N, y):
    """x, then y, of 4.6 GB in 3 slots: the last rows of each slot against their definition."""
    from paper_2605_10670_amd import layer
    g = torch.Generator(device="cuda").manual_seed(30)
    ends = [0, 33, 35000, rows]
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((rows, N), device="cuda")
    w = (torch.randn((3, N, K), generator=g, device="cuda") * K ** -0.5).bfloat16()
    last = [list(range(e - 3, e)) for e in ends[1:]]
    for picked in last:
        x[picked] = torch.randn((3, K), generator=g, device="cuda").bfloat16()
    p = layer.ExpertProduct(num_slots=3, in_features=K, out_features=N, y_dtype=y, max_rows=rows)
    p.run(x, w, out, rows, offset=torch.tensor(ends, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for slot, picked in enumerate(last):
        xd, wd = x[picked].cpu().double(), w[slot].cpu().double()
        lu.check_rounded(out[picked].cpu(), xd @ wd.t(), (xd.abs() @ wd.abs().t()) * (K + 8) * 2.0 ** -23 + 2.0 ** -126)
    p.destroy()


@pytest.mark.parametrize("counts", [(2, 0, 3), (150, 1, 200)])
def test_slots_far_apart(counts):
    """A slot's weights begin past 4 GB of the store."""
    from paper_2605_10670_amd import layer
    c = lu.product_case(31, counts, 512, 128, "fp8", False)
    stride = 2304 << 20
    store = torch.empty(2 * stride + (1 << 20), dtype=torch.uint8, device="cuda")
    size, scales = 512 * 128, 4 * 4
    for s in range(3):
        at = s * stride
        store[at:at + size] = c["w"][s].view(torch.uint8).flatten().cuda()
        store[at + size:at + size + scales] = c["w_scale"][s].contiguous().view(-1).view(torch.uint8).cuda()
    y = torch.empty((c["rows"], 128), device="cuda")
    p = layer.ExpertProduct(num_slots=3, in_features=512, out_features=128, x_dtype="fp8", y_dtype="f32", max_rows=c["rows"],
                            slot_stride=stride, scale_stride=stride)
    p.run(c["x"].cuda(), store.data_ptr(), y, c["rows"], offset=c["offset"].cuda(), x_scale=c["x_scale"].cuda(),
          w_scale=store.data_ptr() + size)
    torch.cuda.synchronize()
    lu.check_product(c, "f32", y.cpu(), None)
    p.destroy()
