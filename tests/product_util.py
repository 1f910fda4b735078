"""Which kernel a product was computed by, for tests that have to reach a certain one."""
import re

import torch

from paper_2605_10670_amd import layer

TORCH_OF = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def kernels_of(call):
    """The product kernels that a call launches, as "few", "thin" or "tiled" with their integer template arguments."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    found = []
    for e in prof.key_averages():
        m = re.search(r"k_product_(\w+)<(.*?)>\(", e.key)
        if m:
            found.append((m[1], tuple(v.strip() for v in m[2].split(","))))
    return found


def form_of(call):
    """"thin", "few M N" (tiles of 16 weight rows and of 16 tokens) or "tiled N" (64 tokens each)."""
    (kind, args), = kernels_of(call)
    return " ".join([kind, *{"thin": (), "few": args[3:5], "tiled": args[-1:]}[kind]])


def run(x, w, offset, y_dtype, gate, x_scale=None, w_scale=None, xt="bf16"):
    """Operands on the GPU through layer.ExpertProduct -> (y, y_scale, form)."""
    P, weight_rows, K = w.shape
    N, rows = weight_rows // (2 if gate else 1), x.shape[0]
    y = torch.full((rows, N), 77.0, device="cuda").to(TORCH_OF[y_dtype])
    y_scale = torch.full((rows, N // 128), 77.0, device="cuda") if y_dtype == "fp8" else None
    product = layer.ExpertProduct(num_slots=P, in_features=K, out_features=N, x_dtype=xt, y_dtype=y_dtype, gate=gate, max_rows=rows)
    form = form_of(lambda: product.run(x, w, y, rows, offset=offset, x_scale=x_scale, w_scale=w_scale, y_scale=y_scale))
    product.destroy()
    return y, y_scale, form
