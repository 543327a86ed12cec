"""A cache held in 8 bits: its append and gather against the definition of the
codes, its attention calls against 64-bit values."""
import ctypes

import numpy as np
import pytest
import torch

import cache8_reference as ref
from cache8_reference import D, PAGE

pytestmark = pytest.mark.gpu
FORMATS = ("int8", "e4m3")


def make(ws, H, pages, fmt, **kw):
    return ws.Cache(H, pages, kv_format=fmt, rope_max_pos=(64, 64, 64), **kw)


def gathered(cache, unit, kind, n, H):
    k, v = (torch.full((n, H, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.gather([dict(unit=unit, kind=kind, k_out=k, v_out=v)])
    return k, v


def hard_blocks(gen, n, H):
    """Values with blocks where a rounding or a scale can go wrong."""
    x = ref.normal(gen, n, H, D).float()
    for h in range(H):
        kind = h % 6
        if kind == 1:
            x[:, h] = 0
        elif kind == 2:  # one outlier per block
            x[::PAGE, h, 5] = 1000.0
        elif kind == 3:  # halves of a power-of-two scale: ties
            x[:, h] = torch.round(x[:, h] * 40).clamp(-126, 126) + 0.5
            x[::PAGE, h, 0] = 127.0
        elif kind == 4:  # far ends of the range
            x[:, h] *= 2.0 ** -130
        elif kind == 5:
            x[:, h] *= 7e37
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n,H,fused", [(1, 1, False), (4, 3, True), (63, 6, False), (64, 2, True), (65, 6, True),
                                       (200, 12, False), (920, 7, True)])
def test_raw_codes_are_exact(ws, fmt, n, H, fused):
    gen = torch.Generator().manual_seed(n * 31 + H)
    k, v = hard_blocks(gen, n, H), hard_blocks(gen, n, H).flip(1)
    if fused:  # column blocks of one projection's output
        both = torch.cat([k, v, k], dim=1).cuda()
        kd, vd = both[:, :H], both[:, H:2 * H]
    else:
        kd, vd = k.cuda(), v.cuda()
    cache = make(ws, H, n // PAGE + 3, fmt)
    cache.append(0, ws.WS_KIND_VIDEO, kd, vd)
    kc, vc, ks, vs = cache.export_codes(0, ws.WS_KIND_VIDEO)
    back = gathered(cache, 0, ws.WS_KIND_VIDEO, n, H)
    host = cache.export(0, ws.WS_KIND_VIDEO)
    for x, codes, scales, got, exported in ((k, kc, ks, back[0], host[0]), (v, vc, vs, back[1], host[1])):
        q, s = ref.quantise(ref.stored(x.double(), fmt), fmt)
        np.testing.assert_array_equal(scales.astype(np.float64), s.numpy())
        np.testing.assert_array_equal(ref.decode(codes, fmt).numpy(), q.numpy())
        want = (q * ref.spread(s, n)).float().to(torch.bfloat16)  # a code times its scale is exact in fp32
        assert torch.equal(got.cpu().view(torch.int16) & 0x7fff, want.view(torch.int16) & 0x7fff)
        assert torch.equal(got.cpu().float(), want.float())
        np.testing.assert_array_equal(exported, got.cpu().view(torch.int16).numpy().view(np.uint16))
    held = all(torch.equal(ref.stored(x.double(), fmt), x.double()) for x in (k, v))
    assert cache.check() == (0 if held else 2)
    cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n,H", [(1, 2), (67, 3), (252, 5)])
def test_normed_and_rotated_keys(ws, fmt, n, H):
    """Keys in fp32 (1e-5 of the block's largest, for norm, products and angles from
    fp32 tables), rounded once: off by at most half a step of the code."""
    gen = torch.Generator().manual_seed(n)
    k, v, pos = ref.normal(gen, n, H, D), ref.normal(gen, n, H, D), ref.positions(9, n)
    gamma = 1 + 0.1 * torch.randn(D, generator=gen)
    cache = make(ws, H, 8, fmt)
    cache.append(9, ws.WS_KIND_AUDIO, k.cuda(), v.cuda(), ws.WS_APPEND_NORM_ROPE, pos.cuda(), gamma.cuda())
    codes, _, scales, _ = cache.export_codes(9, ws.WS_KIND_AUDIO)
    x = ref.norm_rope(k, pos, gamma)
    s = torch.from_numpy(scales).double()
    top = torch.stack([x[b:b + PAGE].abs().amax((0, 2)) for b in range(0, n, PAGE)])
    if fmt == "int8":
        assert ((s * 127 / top - 1).abs() < 1e-5 + 2.0 ** -15).all()
    else:
        assert (top <= 448 * s * (1 + 1e-5)).all() and (top > 224 * s * (1 - 1e-5)).all()
    each = ref.spread(s, n)
    got = ref.decode(codes, fmt) * each
    half = each / 2 if fmt == "int8" else torch.maximum(x.abs() * 2.0 ** -4, each * 2.0 ** -10)
    assert ((got - x).abs() <= half * (1 + 2.0 ** -4) + 1e-5 * ref.spread(top, n)).all()
    cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_non_finite_values_are_stored_as_zero_and_flagged(ws, fmt):
    gen = torch.Generator().manual_seed(3)
    k, v = ref.normal(gen, 70, 2, D), ref.normal(gen, 70, 2, D)
    clean_k, clean_v = k.clone(), v.clone()
    for x, clean, at in ((k, clean_k, (3, 1, 5)), (v, clean_v, (66, 0, 127)), (v, clean_v, (1, 0, 0))):
        x[at] = float("inf") if at[0] == 3 else float("nan") if at[0] == 1 else float("-inf")
        clean[at] = 0
    cache, other = make(ws, 2, 4, fmt), make(ws, 2, 4, fmt)
    cache.append(0, ws.WS_KIND_COND, k.cuda(), v.cuda())
    other.append(0, ws.WS_KIND_COND, clean_k.cuda(), clean_v.cuda())
    for a, b in zip(cache.export_codes(0, ws.WS_KIND_COND), other.export_codes(0, ws.WS_KIND_COND)):
        np.testing.assert_array_equal(a & 0x7f if a.dtype == np.uint8 and fmt == "e4m3" else a,
                                      b & 0x7f if b.dtype == np.uint8 and fmt == "e4m3" else b)
    assert cache.check() == 2 and cache.check() == 0 and other.check() == 0
    cache.close()
    other.close()


@pytest.mark.parametrize("fmt", FORMATS + ("bf16",))
def test_batches_rewrites_and_bounds_of_a_gather(ws, fmt):
    """Ten segments in one append and one gather (two launches each), a rewrite of
    one of them, and the rows around each output left as they were."""
    H, gen = 3, torch.Generator().manual_seed(11)
    lengths = [1, 64, 65, 4, 130, 7, 63, 200, 2, 90]
    cache, alone = make(ws, H, 32, fmt), make(ws, H, 32, fmt)
    data = [(ref.normal(gen, n, H, D).cuda(), ref.normal(gen, n, H, D).cuda()) for n in lengths]
    item = lambda u: dict(unit=u, kind=ws.WS_KIND_VIDEO, k=data[u][0], v=data[u][1])  # noqa: E731
    cache.append_many([item(u) for u in range(10)])
    for u in reversed(range(10)):
        alone.append(**item(u))
    new = (ref.normal(gen, 65, H, D).cuda(), ref.normal(gen, 65, H, D).cuda())
    for c in (cache, alone):
        c.append(2, ws.WS_KIND_VIDEO, *new)
    data[2] = new
    total = sum(lengths) + 2 * len(lengths)
    outs = [torch.full((total, H, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    at, items, spans = 1, [], []
    for u, n in enumerate(lengths):
        items.append(dict(unit=u, kind=ws.WS_KIND_VIDEO, k_out=outs[0][at:at + n], v_out=outs[1][at:at + n]))
        spans.append((at, n))
        at += n + 2
    cache.gather(items)
    for i in range(2):
        kept = torch.ones(total, dtype=torch.bool)
        for u, (lo, n) in enumerate(spans):
            kept[lo:lo + n] = False
            want = gathered(alone, u, ws.WS_KIND_VIDEO, n, H)[i]
            assert torch.equal(outs[i][lo:lo + n], want), (u, i)
            if fmt == "bf16":
                assert torch.equal(want, data[u][i])
        assert (outs[i].cpu()[kept] == 7.0).all()
    only = torch.zeros_like(data[7][0])
    cache.gather([dict(unit=7, kind=ws.WS_KIND_VIDEO, v_out=only)])
    assert torch.equal(only, outs[1][spans[7][0]:spans[7][0] + 200])
    cache.close()
    alone.close()


class Stream8:
    """A stream's cache in 8 bits: slice, units of video and audio tokens; and what
    it stands for, in 64 bits."""

    def __init__(self, ws, fmt, H, cond, units, video, audio, seed=0, std=1.0, max_q=1024, spare=4):
        gen = torch.Generator().manual_seed(seed)
        self.ws, self.H, self.units, self.gen = ws, H, units, gen
        self.video, self.audio = video, audio
        self.gamma = 1 + 0.1 * torch.randn(D, generator=gen)
        pages = -(-max(cond, 1) // PAGE) + units * (-(-max(video, 1) // PAGE) - (-max(audio, 1) // PAGE))
        self.cache = make(ws, H, pages + spare, fmt, max_q_tokens=max_q)
        self.segs, self.order = {}, []
        if cond:
            self.put(0, ws.WS_KIND_COND, cond, std)
        for u in range(units):
            for kind, n in ((ws.WS_KIND_VIDEO, video), (ws.WS_KIND_AUDIO, audio)):
                if n:
                    self.put(u, kind, n, std)

    def put(self, unit, kind, n, std=1.0):
        ws, gen = self.ws, self.gen
        k, v = ref.normal(gen, n, self.H, D, std=std), ref.normal(gen, n, self.H, D)
        if kind == ws.WS_KIND_COND:
            self.cache.append(unit, kind, k.cuda(), v.cuda())
        else:
            self.cache.append(unit, kind, k.cuda(), v.cuda(), ws.WS_APPEND_NORM_ROPE,
                              ref.positions(unit, n).cuda(), (std * self.gamma).cuda())
        self.segs[unit, kind] = [t.double().cpu() for t in gathered(self.cache, unit, kind, n, self.H)]

    def keys(self, unit, kinds, low=-1):
        seen = [s for (u, kind), s in sorted(self.segs.items())
                if kind in kinds and u <= unit and (kind == self.ws.WS_KIND_COND or u >= low)]
        if not seen:
            return [torch.zeros(0, self.H, D, dtype=torch.float64)] * 2
        return torch.cat([s[0] for s in seen]), torch.cat([s[1] for s in seen])

    def queries(self, n, unit):
        q, pos = ref.normal(self.gen, n, self.H, D), ref.positions(unit, n)
        return q, pos, ref.norm_rope(q, pos, self.gamma)


SHAPES = [
    (1, 0, 1, 1, 0, 1, False),       # one key, one row
    (2, 5, 1, 40, 3, 40, False),
    (3, 64, 3, 128, 4, 129, False),  # full pages
    (2, 30, 4, 333, 3, 333, False),
    (5, 0, 2, 65, 0, 257, False),
    (1, 1, 1, 0, 1, 64, True),
    (3, 20, 3, 100, 4, 4, True),
    (2, 100, 9, 70, 5, 17, True),    # several key ranges
    (12, 64, 6, 252, 4, 1, True),
]
# splits: the call's own choice of kernel, or the video kernel's form over 1 or 3 key ranges


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,cond,units,video,audio,rows,few,splits",
                         [(*c, n) for c in SHAPES for n in ((0,) if c[-1] else (0, 1, 3))])
def test_attention_over_8_bits(ws, fmt, H, cond, units, video, audio, rows, few, splits):
    st = Stream8(ws, fmt, H, cond, units, video, audio, seed=rows)
    st.cache.set_option(ws.WS_OPT_VIDEO_KV_SPLITS, splits)
    kinds = (ws.WS_KIND_COND, ws.WS_KIND_VIDEO) + ((ws.WS_KIND_AUDIO,) if few else ())
    q, pos, q64 = st.queries(rows, units - 1)
    call = st.cache.audio_attention if few else st.cache.unit_attention
    k, v = st.keys(units - 1, kinds)
    want, bound = ref.attend(q64, k, v)
    out = torch.full_like(q, float("nan")).cuda()
    call(q.cuda(), out, ws.mask_spec(units - 1, kinds=kinds), positions=pos.cuda(), gamma=st.gamma.cuda())
    ref.check(out, want, bound, "normed in the call")
    qp = torch.empty_like(out)
    st.cache.step_append(queries=[dict(q=q.cuda(), q_out=qp, positions=pos.cuda(), gamma=st.gamma.cuda())])
    call(qp, out, ws.mask_spec(units - 1, kinds=kinds), ws.WS_QUERY_PREPARED)
    ref.check(out, want, bound, "prepared")
    # raw rows in a wider buffer, under a window of units, with a scale
    wide = torch.full((rows + 2, H + 1, D), 3.0, dtype=torch.bfloat16, device="cuda")
    dest = wide[1:rows + 1, :H]
    low = max(0, units - 2)
    call(q.cuda(), dest, ws.mask_spec(units - 1, low, kinds), ws.WS_APPEND_RAW, scale=0.05)
    want, bound = ref.attend(q.double(), *st.keys(units - 1, kinds, low), scale=0.05)
    ref.check(dest, want, bound, "raw")
    assert (wide[0] == 3).all() and (wide[-1] == 3).all() and (wide[:, H] == 3).all()
    # nothing visible
    call(q.cuda(), out, ws.mask_spec(-1, kinds=kinds), ws.WS_APPEND_RAW)
    assert (out == 0).all()
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("running_max", [0, 1])
@pytest.mark.parametrize("splits", [0, 1, 2])
def test_wide_logits(ws, fmt, few, running_max, splits):
    """Logits beyond the fixed shift's reach, and the running maximum forced."""
    st = Stream8(ws, fmt, 2, 10, 3, 150, 4, std=6.0 if not running_max else 1.0, seed=5)
    st.cache.set_option(ws.WS_OPT_VIDEO_KV_SPLITS, splits)
    st.cache.set_option(ws.WS_OPT_VIDEO_RUNNING_MAX, running_max)
    kinds = (ws.WS_KIND_COND, ws.WS_KIND_VIDEO)
    rows = 20 if few else 150
    q, pos, q64 = st.queries(rows, 2)
    out = torch.empty_like(q).cuda()
    (st.cache.audio_attention if few else st.cache.unit_attention)(
        q.cuda(), out, ws.mask_spec(2, kinds=kinds), positions=pos.cuda(), gamma=st.gamma.cuda())
    ref.check(out, *ref.attend(q64, *st.keys(2, kinds)))
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,rows", [(12, 920), (40, 252), (5, 1024)])
def test_long_streams(ws, fmt, heads, rows):
    """More pages than a workgroup's window of list entries, several tiles, heads cut
    by the shares; every head against 64 bits on some rows, the same bits again, and
    the bf16 kernel over what the cache stands for."""
    st = Stream8(ws, fmt, heads, 100, 10, 920, 0, seed=rows)
    kinds = (0, 1)
    k, v = st.keys(9, kinds)
    q = ref.normal(st.gen, rows, heads, D)
    out = torch.full_like(q, float("nan")).cuda()
    mask = ws.mask_spec(9, kinds=kinds)
    st.cache.unit_attention(q.cuda(), out, mask, ws.WS_APPEND_RAW)
    some = torch.randperm(rows, generator=st.gen)[:24]
    ref.check(out[some.cuda()], *ref.attend(q[some].double(), k, v), label="some rows")
    again = torch.empty_like(out)
    st.cache.unit_attention(q.cuda(), again, mask, ws.WS_APPEND_RAW)
    assert torch.equal(out, again)
    plain = make(ws, heads, 10 * 15 + 4, "bf16")
    for (u, kind), (kk, vv) in sorted(st.segs.items()):
        plain.append(u, kind, kk.to(torch.bfloat16).cuda(), vv.to(torch.bfloat16).cuda())
    plain.unit_attention(q.cuda(), again, mask, ws.WS_APPEND_RAW)
    # two of the device's results, each within the bound; their 2-norm like two roundings
    assert (out.float() - again.float()).norm() <= 2 * ref.U * again.float().norm()
    plain.close()
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_groups_of_units(ws, fmt):
    st = Stream8(ws, fmt, 3, 20, 5, 90, 0, seed=2)
    kinds = (ws.WS_KIND_COND, ws.WS_KIND_VIDEO)
    sizes, masks = (90, 0, 33, 200), ((2, 1), (3, 0), (4, 4), (-1, 0))
    rows = sum(sizes)
    q = ref.normal(st.gen, rows, 3, D)
    out = torch.full_like(q, float("nan")).cuda()
    st.cache.unit_attention_groups(q.cuda(), out, [(n, ws.mask_spec(u, lo, kinds if u >= 0 else ()))
                                                   for n, (u, lo) in zip(sizes, masks)], ws.WS_APPEND_RAW)
    at = 0
    for n, (u, lo) in zip(sizes, masks):
        if n and u >= 0:
            ref.check(out[at:at + n], *ref.attend(q[at:at + n].double(), *st.keys(u, kinds, lo)), label=str(u))
        elif n:
            assert (out[at:at + n] == 0).all()
        at += n
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_stream_of_steps(ws, fmt):
    """Append, prepare, attend, commit, evict: units through a window of two, as a
    program runs them; both step entry points; pages taken again."""
    H, n, a = 3, 130, 4
    st = Stream8(ws, fmt, H, 40, 0, n, a, seed=8, spare=8)
    kv, ka = (0, 1), (0, 1, 2)
    for unit in range(5):
        data, items, queries, outs, refs = [], [], [], [], []
        for kind, m in ((ws.WS_KIND_VIDEO, n), (ws.WS_KIND_AUDIO, a)):
            k, v = ref.normal(st.gen, m, H, D).cuda(), ref.normal(st.gen, m, H, D).cuda()
            q, pos, q64 = st.queries(m, unit)
            rope = dict(mode=ws.WS_APPEND_NORM_ROPE, positions=pos.cuda(), gamma=st.gamma.cuda())
            items.append(dict(unit=unit, kind=kind, k=k, v=v, **rope))
            queries.append(dict(q=q.cuda(), q_out=torch.empty_like(k), **rope))
            outs.append([torch.empty_like(k) for _ in range(2)])
            data.append((kind, m))
            refs.append(q64)
        st.cache.step_append(items, queries)
        for i, call in enumerate((st.cache.step_attention, st.cache.step_attention_noalloc)):
            call(*[dict(q=queries[j]["q_out"], out=outs[j][i], mask=ws.mask_spec(unit, unit - 1, kinds),
                        mode=ws.WS_QUERY_PREPARED) for j, kinds in enumerate((kv, ka))])
        for kind, m in data:
            st.segs[unit, kind] = [t.double().cpu() for t in gathered(st.cache, unit, kind, m, H)]
        for j, kinds in enumerate((kv, ka)):
            assert torch.equal(*outs[j])
            ref.check(outs[j][0], *ref.attend(refs[j], *st.keys(unit, kinds, unit - 1)), label=f"{unit} {kinds}")
        st.cache.commit(unit)
        with pytest.raises(ws.WsError):
            st.cache.step_append(items, queries)
        st.cache.evict_before(unit)
        st.segs = {key: s for key, s in st.segs.items() if key[0] >= unit or key[1] == 0}
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_other_streams_and_graph_replays(ws, fmt):
    """A step captured into a graph, on a stream of its own, replayed between eager
    calls on other inputs: every replay gives the eager result."""
    H, n = 2, 100
    st = Stream8(ws, fmt, H, 30, 2, n, 0, seed=4)
    k, v, q = (ref.normal(st.gen, n, H, D).cuda() for _ in range(3))
    other = [ref.normal(st.gen, n, H, D).cuda() for _ in range(3)]
    out, eager, ko, vo = (torch.empty_like(q) for _ in range(4))
    mask = ws.mask_spec(1, kinds=(0, 1))

    def step(k, v, q, out):
        st.cache.append(1, ws.WS_KIND_VIDEO, k, v)
        st.cache.unit_attention(q, out, mask, ws.WS_APPEND_RAW)
        st.cache.gather([dict(unit=1, kind=ws.WS_KIND_VIDEO, k_out=ko, v_out=vo)])

    step(k, v, q, eager)
    torch.cuda.synchronize()
    kept = [t.clone() for t in (eager, ko, vo)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(k, v, q, out)
    for i in range(4):
        if i:
            step(*other, eager)
            torch.cuda.synchronize()
            assert not torch.equal(eager, kept[0])
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, kept[0]) and torch.equal(ko, kept[1]) and torch.equal(vo, kept[2]), i
    with torch.cuda.stream(stream):
        step(*other, out)
    torch.cuda.synchronize()
    assert torch.equal(out, eager) if i else True
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_block_step_over_8_bits(ws, fmt):
    """The sub-block's step takes an 8-bit cache: its attention output is that of
    the same projections' rows."""
    H, n, a, hid = 2, 70, 4, 2 * D
    st = Stream8(ws, fmt, H, 20, 1, n, a, seed=6)
    g = torch.Generator().manual_seed(1)
    x = ref.normal(g, n + a, hid).cuda()
    w_qkv, w_out = ref.normal(g, hid, 3 * hid, std=hid ** -0.5).cuda(), ref.normal(g, hid, hid, std=hid ** -0.5).cuda()
    block = ws.Block(st.cache, w_qkv, w_out, n + a)
    y, o = torch.empty_like(x), torch.empty_like(x)
    pv, pa = ref.positions(1, n), ref.positions(1, a)
    ones = torch.ones(D, device="cuda")
    block.step(x, n, 1, pv.cuda(), pa.cuda(), ones, ones, y, ws.mask_spec(1, kinds=(0, 1)),
               ws.mask_spec(1, kinds=(0, 1, 2)), attn_out=o)
    for kind, m in ((1, n), (2, a)):
        st.segs[1, kind] = [t.double().cpu() for t in gathered(st.cache, 1, kind, m, H)]
    # the projection's bf16 rows: half a step of each off the 64-bit ones, which moves a
    # logit of unit-scale rows by a few 2^-8; four times the bound of exact rows
    qkv = (x.cpu().float() @ w_qkv.cpu().float()).to(torch.bfloat16).view(n + a, 3, H, D)
    for rows, pos, kinds in ((slice(0, n), pv, (0, 1)), (slice(n, n + a), pa, (0, 1, 2))):
        q64 = ref.norm_rope(qkv[rows, 0], pos, torch.ones(D))
        want, bound = ref.attend(q64, *st.keys(1, kinds))
        ref.check(o.view(n + a, H, D)[rows], want, 4 * bound, str(kinds))
    block.close()
    st.cache.close()


def test_refusals(ws):
    with pytest.raises(ValueError):
        ws.Cache(2, 4, kv_format="fp8")
    cfg = ws.ws_cache_config()
    cfg.num_heads, cfg.head_dim, cfg.page_tokens, cfg.max_pages, cfg.max_q_tokens = 2, 128, 64, 4, 64
    cfg.rope_max_pos[:], cfg.rope_pairs[:], cfg.rope_theta = [4, 4, 4], [22, 21, 21], 1e4
    for fmt in (-1, 3):
        with pytest.raises(ws.WsError) as e:
            ws.ws_cache_create_format(cfg, fmt)
        assert e.value.status == ws.WS_ERR_INVALID_ARG
    cache, plain = make(ws, 2, 4, "int8"), make(ws, 2, 4, "bf16")
    assert ws.ws_cache_format(cache.handle) == ws.WS_KV_INT8 and ws.ws_cache_format(plain.handle) == ws.WS_KV_BF16
    x = torch.zeros(70, 2, D, dtype=torch.bfloat16, device="cuda")
    cache.append(0, 1, x, x)
    plain.append(0, 1, x, x)

    def status(fn, *args, **kw):
        with pytest.raises(ws.WsError) as e:
            fn(*args, **kw)
        return e.value.status

    assert status(plain.export_codes, 0, 1) == ws.WS_ERR_UNSUPPORTED
    assert status(cache.export_codes, 1, 1) == ws.WS_ERR_UNKNOWN_UNIT
    out = torch.empty_like(x)
    p = out.data_ptr()

    def gather(*items):
        return status(ws.ws_kv_gather, cache.handle, [ws.ws_gather_item(*i) for i in items], 0)

    assert gather() == ws.WS_ERR_INVALID_ARG
    assert gather(*[(0, 1, 70, p, None, 256, 128)] * 17) == ws.WS_ERR_INVALID_ARG
    assert gather((0, 3, 70, p, None, 256, 128)) == ws.WS_ERR_INVALID_ARG
    assert gather((0, 1, 70, p, None, 256, 128), (0, 2, 70, p, None, 256, 128)) == ws.WS_ERR_UNKNOWN_UNIT
    assert gather((0, 1, 69, p, None, 256, 128)) == ws.WS_ERR_SHAPE
    assert gather((0, 1, 70, None, None, 256, 128)) == ws.WS_ERR_INVALID_ARG
    assert gather((0, 1, 70, p + 2, None, 256, 128)) == ws.WS_ERR_INVALID_ARG
    assert gather((0, 1, 70, p, p, 252, 128)) == ws.WS_ERR_INVALID_ARG
    assert gather((0, 1, 70, p, None, 64, 128)) == ws.WS_ERR_INVALID_ARG
    with pytest.raises(ws.WsError):
        cache.gather([])
    with pytest.raises(ws.WsError):
        cache.gather([dict(unit=0, kind=1, k_out=out[:69])])
    with pytest.raises(ValueError):
        cache.gather([dict(unit=0, kind=1, k_out=out, v_out=torch.empty(70, 4, D, dtype=torch.bfloat16,
                                                                        device="cuda")[:, :2])])
    # out of pages: nothing of the batch is taken
    big = torch.zeros(200, 2, D, dtype=torch.bfloat16, device="cuda")
    assert status(cache.append_many, [dict(unit=1, kind=1, k=x, v=x), dict(unit=2, kind=1, k=big, v=big)]) == \
        ws.WS_ERR_OUT_OF_PAGES
    assert cache.info().pages_free == 2 and cache.info().n_segments == 1
    cache.close()
    plain.close()
