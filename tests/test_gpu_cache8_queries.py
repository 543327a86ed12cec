"""Many rows over 8-bit pages where the queries' own rounding is felt: dims that differ
by many powers of two, in queries and (the other way round) in keys, rows of zeros, rows
and keys far from 1."""
import pytest
import torch

import cache8_reference as ref
from cache8_reference import D, U

pytestmark = pytest.mark.gpu


def attend_wide(q, k, v, scale):
    """ref.attend, and what the queries' two e4m3 terms move an output by beside it: a
    query errs by 2^-8 of itself (U) or 2^-21 of the row's largest, so a logit by
    scale (U sum |q k| + 2^-21 max |q| sum |k|), and an output by the weights' mean of that
    times |v| + |o|."""
    out, bound = ref.attend(q, k, v, scale=scale)
    for h in range(q.shape[1]):
        qa, ka = q[:, h].abs(), k[:, h].abs()
        p = torch.softmax(scale * (q[:, h] @ k[:, h].T), 1)
        w = p * scale * (U * (qa @ ka.T) + 2.0 ** -21 * qa.amax(1, keepdim=True) * ka.sum(1))
        bound[:, h] += 1.05 * (w @ v[:, h].abs() + out[:, h].abs() * w.sum(1, keepdim=True))
    return out, bound


@pytest.mark.parametrize("fmt", ("e4m3", "int8"))
@pytest.mark.parametrize("rows,tokens,spread,shift", [
    (300, 200, 0, 0), (300, 200, 8, 0), (150, 65, 13, 0),
    (600, 130, 4, 60), (257, 64, 4, -60), (70, 300, 6, 100)])
def test_queries_of_a_wide_range(ws, fmt, rows, tokens, spread, shift):
    """Dim d of the queries carries 2^-a[d] 2^-shift, of the keys 2^(a[d] - spread) 2^shift."""
    gen = torch.Generator().manual_seed(rows + spread)
    H = 3
    a = torch.randint(0, spread + 1, (H, D), generator=gen).float()
    q = (torch.randn(rows, H, D, generator=gen) * 2.0 ** (-a - shift)).to(torch.bfloat16)
    q[rows // 2] = 0
    x = torch.randn(tokens, H, D, generator=gen)
    k = (x * 2.0 ** (a - spread + shift)).to(torch.bfloat16)
    v = ref.normal(gen, tokens, H, D)
    scale = 2.0 ** (spread - 4)  # logits of about 1 whatever the spread
    cache = ws.Cache(H, 16, kv_format=fmt, rope_max_pos=(64, 64, 64))
    cache.set_option(ws.WS_OPT_VIDEO_KV_SPLITS, 1)  # the many-row form
    cache.append(0, ws.WS_KIND_VIDEO, k.cuda(), v.cuda(), ws.WS_APPEND_RAW)
    codes = cache.export_codes(0, ws.WS_KIND_VIDEO)
    kk, vv = (ref.decode(c, fmt) * ref.spread(torch.from_numpy(s).double(), tokens)
              for c, s in ((codes[0], codes[2]), (codes[1], codes[3])))
    bf = lambda t: t.to(torch.bfloat16).double()  # what the attention reads
    out = torch.full_like(q, float("nan")).cuda()
    cache.unit_attention(q.cuda(), out, ws.mask_spec(0, kinds=(ws.WS_KIND_VIDEO,)), ws.WS_APPEND_RAW, scale=scale)
    ref.check(out, *attend_wide(q.double(), bf(kk), bf(vv), scale))
    cache.close()
