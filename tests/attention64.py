"""Attention of many query rows in 64 bits, one row at a time by its definition, and how far a kernel may be from it."""
import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}        # finfo(t).eps / 2


def attend(Q, K, V, seen, scale=None):
    """Q [n, Hq, D], K and V [Hkv, m, D], seen [n, m] truth values -> (O, weights times |V|, largest sum of |q||k| of a row, scaled),
    each [n, Hq, ...], float64.  What a row does not see is left out, not multiplied by zero."""
    n, Hq, D = Q.shape
    Hkv, m, _ = K.shape
    scale = D ** -0.5 if scale is None else scale
    if m == 0 or n == 0:
        nothing = torch.zeros((n, Hq, D), dtype=torch.float64, device=Q.device)
        return nothing, nothing, nothing[..., :1]
    q = Q.double().view(n, Hkv, Hq // Hkv, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
    k, v = K.double(), V.double()
    rows = seen.repeat(Hq // Hkv, 1)
    s = torch.stack([q[h] @ k[h].t().contiguous() for h in range(Hkv)]) * scale
    s = torch.where(rows[None], s, torch.tensor(-torch.inf, dtype=torch.float64, device=Q.device))
    top = s.max(-1, keepdim=True).values
    w = torch.exp(s - torch.where(top == -torch.inf, torch.zeros_like(top), top))
    w = torch.where(rows[None], w, torch.zeros_like(w))
    total = w.sum(-1, keepdim=True)
    w = torch.where(total == 0, w, w / total)
    plain = torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0)
    o = torch.stack([w[h] @ plain[h] for h in range(Hkv)])
    size = torch.stack([w[h] @ plain[h].abs() for h in range(Hkv)])
    for h, j, d in (~torch.isfinite(v)).nonzero().tolist():               # few: row by row
        o[h, :, d] += torch.where(rows[:, j], w[h, :, j] * v[h, j, d], 0.0)
    big = torch.stack([q[h].abs() @ torch.nan_to_num(k[h], nan=0.0, posinf=0.0, neginf=0.0).abs().t().contiguous() for h in range(Hkv)]) * scale
    big = torch.where(rows[None], big, 0.0).amax(-1)

    def back(x):
        return x.view(Hkv, Hq // Hkv, n, -1).permute(2, 0, 1, 3).reshape(n, Hq, -1)
    return back(o), back(size), back(big)


def allowed(dtype, o, size, big, m, D):
    """Off by at most: scores, sums of D products in fp32 times the scale, (D + 4) roundings of at most `big` each, for the key and for the
    maximum; the exponential and the sums over m keys, m + 8 roundings; for bf16 the rounding of every weight, in the sum over
    values and in the sum of weights; all relative to `size`.  Then the rounding of the result."""
    weights = 2 * (D + 4) * 2.0 ** -24 * big + (m + 8) * 2.0 ** -23
    if dtype == torch.bfloat16:
        weights = weights + 2 * HALF_STEP[dtype]
    return size * weights + HALF_STEP[dtype] * o.abs() + 1e-30


def check(got, want, m):
    o, size, big = want
    D = got.shape[-1]
    tol = allowed(got.dtype, o, size, big, m, D)
    off = (got.double() - o).abs()
    finite = torch.isfinite(o)
    assert torch.equal(torch.isfinite(got), finite), "not finite in other places"
    if got.numel() == 0:
        return
    worst = torch.where(finite, off / tol, 0.0).max().item()
    assert worst <= 1.0, "%.3g times what rounding allows" % worst
