"""Plain implementations in 64 bits of the operators around the paged cache, and the error bounds of the kernels' arithmetic."""
import math

import torch

HALF_STEP = 2.0 ** -8          # a value rounded to bf16 is off by at most this, relative to it


def causal(q, k, v, context, scale=None, rows=None):
    """q [n][Hq][D], k, v [context + n][Hkv][D] (bf16): (out, bound), the causal attention of tokens context .. in fp64 and, for
    every value, how far the kernels' bf16 output may be off.  rows: only these tokens of q.

    The bound: with w the softmax weights and A = sum w |v|,
      - P is rounded to bf16 for the product with V, its sum is not:                      2^-8 A
      - a score is an fp32 sum of D products: off by d_s <= (D + 4) 2^-24 scale sum |q k|, and its exponential by a factor
        2^e with 2^-12 for the exponential itself; numerator and denominator:              2 (d_s + 2^-12) A
      - fp32 accumulation of the products and the sum, in blocks of 128 keys:              2 (128 + tiles) 2^-24 A
      - the output is rounded to bf16:                                                   2^-8 |out|  (+ the smallest normal number)
    """
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = scale or 1.0 / math.sqrt(d)
    token = torch.arange(n, device=q.device) if rows is None else torch.as_tensor(rows, device=q.device)
    key = torch.arange(k.shape[0], device=q.device)
    hidden = key[None, :] > context + token[:, None]
    out, bound = [], []
    for h in range(hq):
        qh, kh, vh = q[token, h].double(), k[:, h // g].double(), v[:, h // g].double()
        x = (qh @ kh.T * scale).masked_fill(hidden, -math.inf)
        w = torch.softmax(x, dim=1)
        size = (qh.abs() @ kh.abs().T * scale).masked_fill(hidden, 0.0).amax(dim=1, keepdim=True)
        o, a = w @ vh, w @ vh.abs()
        rel = HALF_STEP + 2 * ((d + 4) * 2.0 ** -24 * size + 2.0 ** -12) + 2 * (128 + k.shape[0] / 128) * 2.0 ** -24
        out.append(o)
        bound.append(rel * a + HALF_STEP * o.abs() + 2.0 ** -126)
    return torch.stack(out, dim=1), torch.stack(bound, dim=1)


def rope_table(n_positions, rot, base=10000.0, device="cuda"):
    """fp32 [positions][rot]: cosines, then sines."""
    freq = base ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))
    angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * freq[None, :]
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().to(device)


def rotate(x, rows, interleaved):
    """x [n][H][D] rotated by table rows [n][rot] in fp64: (result, bound).  Two fp32 products and a sum, then a rounding to bf16."""
    rot = rows.shape[1]
    y, size = x.double().clone(), x.double().abs().clone()
    cos, sin = (t[:, None, :].double() for t in rows.chunk(2, dim=1))
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i].double(), x[..., j].double()
    y[..., i], y[..., j] = a * cos - b * sin, b * cos + a * sin
    size[..., i], size[..., j] = (a * cos).abs() + (b * sin).abs(), (b * cos).abs() + (a * sin).abs()
    bound = HALF_STEP * y.abs() + 2.0 ** -22 * size + 2.0 ** -126
    bound[..., rot:] = 0.0                                   # copied
    return y, bound


def check(got, want, bound):
    got = got.double()
    assert torch.isfinite(got).all()
    over = ((got - want).abs() / bound).max().item()
    assert over <= 1.0, f"error {over:.3f} times its bound"
