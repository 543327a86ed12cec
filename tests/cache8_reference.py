"""Plain 64-bit forms of the 8-bit cache and of token windows, for their tests:
written from the definitions, on the CPU, with no code of the product."""
import numpy as np
import torch

PAGE, D, PAIRS, THETA = 64, 128, (22, 21, 21), 10000.0
# bf16: a rounding is off by at most half a step, 2^-8 of the value
U = 2.0 ** -8


def normal(gen, *shape, std=1.0):
    """bf16 values."""
    return (std * torch.randn(*shape, generator=gen)).to(torch.bfloat16)


def positions(unit, n, cols=7):
    i = torch.arange(n, dtype=torch.int32)
    return torch.stack([torch.full_like(i, unit), i // cols, i % cols], dim=1).contiguous()


def norm_rope(x, pos, gamma, eps=1e-6):
    x = x.double()
    x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * gamma.double()
    ang = torch.cat([pos[:, b:b + 1].double() * THETA ** (-torch.arange(n, dtype=torch.float64) / n)
                     for b, n in enumerate(PAIRS)], dim=1)[:, None, :]
    y = torch.empty_like(x)
    y[..., 0::2] = x[..., 0::2] * ang.cos() - x[..., 1::2] * ang.sin()
    y[..., 1::2] = x[..., 0::2] * ang.sin() + x[..., 1::2] * ang.cos()
    return y


def scale_of(a, fmt):
    """The scale of a block with largest magnitude a (float64 of an fp32 value)."""
    if fmt == "int8":
        s = np.float32(np.float32(a) / np.float32(127))
        m, e = np.frexp(np.float64(s))  # rounded up to 16 significant bits
        s = np.ldexp(np.ceil(np.ldexp(m, 16)), int(e) - 16)
        return max(float(s), 2.0 ** -126)
    e = -126
    while a > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def round_e4m3(y):
    step = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def stored(x, fmt):
    """x without the values an 8-bit cache does not hold (0 in their place)."""
    return x.masked_fill(~(x.abs() < (2.0 ** 118 if fmt == "int8" else torch.inf)), 0)


def quantise(x, fmt):
    """[n, H, D] values -> (quotients as the codes stand for them, scales
    [blocks, H]); x in float64."""
    n, H, _ = x.shape
    q, scales = torch.empty_like(x), torch.empty(-(-n // PAGE), H, dtype=torch.float64)
    for b in range(-(-n // PAGE)):
        for h in range(H):
            t = x[b * PAGE:(b + 1) * PAGE, h]
            s = scale_of(float(t.abs().max()), fmt)
            scales[b, h] = s
            y = t / s
            q[b * PAGE:(b + 1) * PAGE, h] = torch.round(y) if fmt == "int8" else round_e4m3(y)
    return q, scales


def spread(scales, n):
    """Scales of the blocks as [n, H, 1]."""
    return scales.repeat_interleave(PAGE, dim=0)[:n, :, None]


def decode(codes, fmt):
    """Stored codes (uint8) as the quotients they stand for."""
    t = torch.from_numpy(codes)
    return (t.view(torch.int8) if fmt == "int8" else t.view(torch.float8_e4m3fn).float()).double()


def attend(q, k, v, see=None, scale=D ** -0.5):
    """softmax(scale q k^T) v per head over the keys that see [rows, keys] leaves,
    a row without any: 0.  q, k, v float64 [*, H, D].  Returns the output and a
    first-order bound on what the device's roundings move it by, elementwise:
      Q'' rounded to bf16       a logit errs by U s sum |q k|
      weights rounded to bf16   U of each, in the sum over values and in the row sum
      bf16 output               U
      fp32 sums of n terms      n 2^-24 in products and in sums; key-range partials
    and 5% for the second-order terms."""
    out, bound = torch.zeros_like(q), torch.zeros_like(q)
    n = k.shape[0]
    for h in range(q.shape[1]):
        s = scale * (q[:, h] @ k[:, h].T)
        if see is not None:
            s = s.masked_fill(~see, -torch.inf)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
        kk, vv = k[:, h], v[:, h]
        if see is not None:  # what no row sees must not matter, whatever it holds
            gone = ~see.any(0)
            kk, vv = kk.masked_fill(gone[:, None], 0), vv.masked_fill(gone[:, None], 0)
        o = p @ vv
        a = p @ vv.abs()
        w = p * (U * scale * (q[:, h].abs() @ kk.abs().T) + U)
        out[:, h] = o
        bound[:, h] = 1.05 * ((2 * U + 4 * n * 2.0 ** -24) * a + w @ vv.abs() + o.abs() * w.sum(1, keepdim=True)) + 1e-30
    return out, bound


def window_mask(n, t0, rows, window, sinks, causal):
    t = torch.arange(t0, t0 + rows)[:, None]
    j = torch.arange(n)[None, :]
    see = (j < sinks) if window == 0 else (j > t - window) | (j < sinks)
    if window == 0:
        see = torch.ones(rows, n, dtype=torch.bool)
    return see & (j <= t) if causal else see.expand(rows, n)


def check(got, ref, bound, label=""):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{label}: not finite"
    ratio = ((got - ref).abs() / bound).max()
    assert ratio <= 1, f"{label}: {float(ratio)} of the bound"
