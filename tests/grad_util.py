"""64-bit statements of the layer's gradients and bounds of what fp32 may be off, for the GPU tests.

U is half a step of fp32.  A sum's bound is (additions on the longest path) * U * the sum of magnitudes."""
import torch

import layer_util as lu

U = 2.0 ** -24
TINY = 2.0 ** -126  # (what a matrix core or an exponential may cut off)
TORCH_OF = lu.TORCH_OF
SENTINEL = 77.0
# additions on the longest path of a row's sum in the norms' kernels: 8 vectors of 8 a lane, 6 steps across lanes, 16 wavefronts
ROW_DEPTH = 64 + 6 + 16


def centred_rows(h, e_h, centred):
    """d (h, or h less its mean) and what fp32 may be off in it; e_h: what h itself is off."""
    if not centred:
        return h, e_h
    d = h - h.mean(dim=1, keepdim=True)
    # the mean is taken out twice: what the first leaves off (ROW_DEPTH + 2) U of mean|h|, is gone after the second but for roundings
    # of about |d| and ROW_DEPTH U of mean|d|; h's own errors pass, and their mean
    first = (ROW_DEPTH + 2) * U * h.abs().mean(dim=1, keepdim=True)
    e = e_h + e_h.mean(dim=1, keepdim=True) + 3 * U * (d.abs() + first) + (ROW_DEPTH + 4) * U * (d.abs().mean(dim=1, keepdim=True) + first)
    return d, e


def root_of(d, e_d, epsilon):
    """sqrt(mean(d^2) + epsilon) and its relative error: of the squares' sum, of d (in the 2-norm), of the root and quotient."""
    root = (d.square().mean(dim=1, keepdim=True) + epsilon).sqrt()
    return root, e_d.square().mean(dim=1, keepdim=True).sqrt() / root + (ROW_DEPTH / 2 + 6) * U


def layer_norm(x, residual, gain, bias, epsilon):
    """(h, y, error of y before its rounding) in 64 bits."""
    h = x.double() + (0 if residual is None else residual.double())
    d, e_d = centred_rows(h, U * h.abs(), True)
    root, rel = root_of(d, e_d, epsilon)
    g = gain.double()
    y = d / root * g
    err = (e_d / root + (d / root).abs() * (rel + 3 * U)) * g.abs()
    if bias is not None:
        y = y + bias.double()
    return h, y, err + U * y.abs() + 2.0 ** -149


def norm_grad(h, gain, grad_y, grad_sum, centred, epsilon):
    """dict of (exact, error before its rounding) for grad_h, grad_gain, grad_bias."""
    h, grad, g = h.double(), grad_y.double(), gain.double()
    T = h.shape[0]
    d, e_d = centred_rows(h, torch.zeros_like(h), centred)
    root, rel = root_of(d, e_d, epsilon)
    u, v = d / root, grad * g
    e_u = e_d / root + u.abs() * (rel + 2 * U)
    along = (v * u).mean(dim=1, keepdim=True)
    e_along = (v.abs() * e_u).mean(dim=1, keepdim=True) + (ROW_DEPTH + 4) * U * (v * u).abs().mean(dim=1, keepdim=True)
    pre = v - u * along
    e_pre = U * v.abs() + e_u * along.abs() + u.abs() * e_along + U * pre.abs()
    if centred:
        mean = v.mean(dim=1, keepdim=True)
        pre = pre - mean
        e_pre = e_pre + (ROW_DEPTH + 3) * U * v.abs().mean(dim=1, keepdim=True) + U * pre.abs()
    out = pre / root
    e_out = e_pre / root + out.abs() * (rel + 3 * U)
    if grad_sum is not None:
        out = out + grad_sum.double()
        e_out = e_out + U * out.abs()
    # over the rows: at most T additions
    r = dict(grad_h=(out, e_out + 2.0 ** -149))
    r["grad_gain"] = ((grad * u).sum(dim=0), (grad.abs() * e_u).sum(dim=0) + (T + 2) * U * (grad * u).abs().sum(dim=0))
    r["grad_bias"] = (grad.sum(dim=0), T * U * grad.abs().sum(dim=0))
    return r


def gate_grad(grad_y, sums):
    """(grad_sums in 64 bits, error before its rounding)."""
    grad, (a, b) = grad_y.double(), sums.double().chunk(2, dim=1)
    s, rest = torch.sigmoid(a), torch.sigmoid(-a)
    of_a, of_b = grad * b * s * (1 + a * rest), grad * a * s
    # the exponential 2 U, a sum, a quotient and a product each: s and rest 6 U; then the products
    e_a = (grad * b).abs() * s * ((a * rest).abs() * 9 * U + (1 + a * rest).abs() * 10 * U)
    e_b = of_b.abs() * 10 * U
    # (an exponential below fp32's normal numbers has no relative precision)
    tiny = 2.0 ** -148 * (1 + a.abs())
    return torch.cat([of_a, of_b], dim=1), torch.cat([e_a + (grad * b).abs() * tiny, e_b + grad.abs() * tiny], dim=1) + 2.0 ** -149


def product_grads(g, x, w, offset, old=None):
    """grad_x and grad_w (exact, error) of g [rows, N], x [rows, K], w [P, N, K] by the offsets (a list); None operands are left out."""
    P = len(offset) - 1
    out = {}
    g = g.double()
    if w is not None:
        wd = w.double()
        e = torch.zeros((g.shape[0], w.shape[2]), dtype=torch.float64)
        m = torch.zeros_like(e)
        for p in range(P):
            at = slice(offset[p], offset[p + 1])
            e[at] = g[at] @ wd[p]
            m[at] = g[at].abs() @ wd[p].abs()
        out["grad_x"] = (e, m * (w.shape[1] + 8) * 2 * U + TINY)
    if x is not None:
        xd = x.double()
        e = torch.zeros((P, g.shape[1], x.shape[1]), dtype=torch.float64)
        m = torch.zeros_like(e)
        for p in range(P):
            at = slice(offset[p], offset[p + 1])
            n = max(0, offset[p + 1] - offset[p])
            if n:
                e[p] = g[at].t() @ xd[at]
                m[p] = g[at].abs().t() @ xd[at].abs() * (n + 8)
        err = m * 2 * U
        if old is not None:
            e = e + old.double()
            err = err + U * e.abs()
        out["grad_w"] = (e, err + TINY)
    return out


def route_grad(topk_idx, topk_w, grad_w, E, logits=None):
    """(grad_logits in 64 bits, error before its rounding)."""
    T, k = topk_idx.shape
    w, gw = topk_w.double(), grad_w.double()
    idx = topk_idx.long()
    chosen = (idx >= 0) & (idx < E)
    w = torch.where(idx >= 0, w, 0.0)
    inner, size = (w * gw).sum(dim=1, keepdim=True), (w * gw).abs().sum(dim=1, keepdim=True)
    e_inner = (k + 2) * U * size
    grad = torch.zeros((T, E), dtype=torch.float64)
    err = torch.zeros_like(grad)
    if logits is None:
        each, e_each = w * (gw - inner), w * (e_inner + 2 * U * (gw.abs() + inner.abs()))
    else:
        v = logits.double()
        v = torch.where(v.isnan(), -torch.inf, v)
        top = v.max(dim=1, keepdim=True).values
        below = torch.where(v == top, 0.0, v - top)
        p = torch.where(v > -torch.inf, below.exp(), 0.0)
        p = p / p.sum(dim=1, keepdim=True).clamp(min=1e-300)
        # the exponential's argument is off by U of itself, its result 2 U, the sum up to 64 + 6 additions
        rel = torch.where(v > -torch.inf, below.abs(), 0.0)
        rel = (rel + (p * rel).sum(dim=1, keepdim=True) + 2 * 2 + 64 + 6 + 2) * U
        grad, err = -p * inner, p * (inner.abs() * rel + e_inner) + 2.0 ** -148 * size
        each, e_each = w * gw, U * (w * gw).abs()
    for j in range(k):
        t = chosen[:, j].nonzero().flatten()
        grad[t, idx[t, j]] += each[t, j]
        err[t, idx[t, j]] += e_each[t, j]
    return grad, err + U * grad.abs() + 2.0 ** -149


def check(name, got, exact, err):
    try:
        lu.check_rounded(got.cpu(), exact, err)
    except AssertionError as e:
        raise AssertionError(f"{name}: {e}") from None
