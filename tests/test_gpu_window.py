"""Attention under a token window with sinks, over caches of every format, against
64-bit values."""
import pytest
import torch

import cache8_reference as ref
from cache8_reference import D
from test_gpu_cache8 import Stream8, gathered

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "int8", "e4m3")


def run(ws, st, q, spec, **kw):
    out = torch.full_like(q, float("nan")).cuda()
    st.cache.window_attention(q.cuda(), out, spec, ws.WS_APPEND_RAW, **kw)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,splits", [(1, 0), (4, 0), (16, 0), (17, 0), (64, 0), (65, 0), (200, 0),
                                         (3, 1), (64, 2), (130, 3), (257, 1), (300, 2)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 64), (64, 0), (100, 3), (130, 65), (0, 0), (1000, 7)])
def test_windows_and_sinks(ws, fmt, rows, splits, window, sinks):
    """Timeline: a 37-token slice, three units of 90 and 3 tokens (pages that end
    inside a tile), rows at its end, from its start, across it and past it; the call's
    own choice of kernel, or the video kernel's form over forced key ranges."""
    st = Stream8(ws, fmt, 2, 37, 3, 90, 3, seed=rows * 7 + window)
    st.cache.set_option(ws.WS_OPT_VIDEO_KV_SPLITS, splits)
    kinds = (0, 1, 2)
    k, v = st.keys(2, kinds)
    n = k.shape[0]
    q = ref.normal(st.gen, rows, 2, D)
    for causal in (True, False):
        for start in (ws.WS_WINDOW_AT_END, 0, 60, n - 1, n + 40):
            spec = ws.window_spec(2, window, sinks, causal=causal, q_start=start, kinds=kinds)
            t0 = n - rows if start == ws.WS_WINDOW_AT_END else start
            see = ref.window_mask(n, t0, rows, window, sinks, causal)
            out = run(ws, st, q, spec)
            ref.check(out, *ref.attend(q.double(), k, v, see), label=f"causal {causal}, start {start}")
            empty = ~see.any(1)
            assert (out.cpu()[empty] == 0).all()
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows", [3, 300])
def test_query_modes_and_unit_windows(ws, fmt, rows):
    """Rows normed in the call or prepared, a mask that hides units and kinds, and
    an order of appends other than the timeline's."""
    st = Stream8(ws, fmt, 3, 0, 4, 75, 5, seed=rows)
    st.put(0, ws.WS_KIND_COND, 50)  # appended last, first in the timeline
    kinds = (0, 1)
    q, pos, q64 = st.queries(rows, 3)
    k, v = st.keys(3, kinds, 2)
    n = k.shape[0]
    want = ref.attend(q64, k, v, ref.window_mask(n, n - rows, rows, 40, 10, True))
    spec = ws.window_spec(3, 40, 10, min_visible_unit=2, kinds=kinds)
    out = torch.full_like(q, float("nan")).cuda()
    st.cache.window_attention(q.cuda(), out, spec, positions=pos.cuda(), gamma=st.gamma.cuda())
    ref.check(out, *want)
    qp = torch.empty_like(out)
    st.cache.step_append(queries=[dict(q=q.cuda(), q_out=qp, positions=pos.cuda(), gamma=st.gamma.cuda())])
    st.cache.window_attention(qp, out, spec, ws.WS_QUERY_PREPARED)
    ref.check(out, *want)
    # no key at all
    st.cache.window_attention(qp, out, ws.window_spec(-1, 40, 10, kinds=kinds), ws.WS_QUERY_PREPARED)
    assert (out == 0).all()
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows", [5, 140])
@pytest.mark.parametrize("running_max", [0, 1])
@pytest.mark.parametrize("splits", [0, 1, 2])
def test_wide_logits(ws, fmt, rows, running_max, splits):
    """Rows under a running maximum, whose first visible keys come late: logits far
    from 0 on either side."""
    st = Stream8(ws, fmt, 2, 20, 3, 200, 0, std=1.0 if running_max else 6.0, seed=rows)
    st.cache.set_option(ws.WS_OPT_VIDEO_KV_SPLITS, splits)
    st.cache.set_option(ws.WS_OPT_VIDEO_RUNNING_MAX, running_max)
    k, v = st.keys(2, (0, 1))
    n = k.shape[0]
    q = ref.normal(st.gen, rows, 2, D)
    for shift in (0.0, 12.0):  # keys near +-q: logits around +-12 sqrt(128)
        for sign in (1, -1):
            qq = (q.float() + sign * shift).to(torch.bfloat16)
            for window, sinks in ((30, 0), (100, 40)):
                out = run(ws, st, qq, ws.window_spec(2, window, sinks))
                see = ref.window_mask(n, n - rows, rows, window, sinks, True)
                ref.check(out, *ref.attend(qq.double(), k, v, see), label=f"{shift * sign} {window}")
    st.cache.close()


@pytest.mark.parametrize("rows", [6, 150])
@pytest.mark.parametrize("bad", ["k", "v", "both"])
@pytest.mark.parametrize("splits", [0, 1, 2])
def test_hidden_infinities_and_nans(ws, rows, bad, splits):
    """Values of any kind in tokens that a row does not see do not reach it, in pages
    that it sees part of (a bf16 cache; an 8-bit one stores none)."""
    gen = torch.Generator().manual_seed(rows)
    H, n = 2, 260
    cache = ws.Cache(H, 8, rope_max_pos=(8, 8, 8))
    cache.set_option(ws.WS_OPT_VIDEO_KV_SPLITS, splits)
    k, v, q = (ref.normal(gen, n, H, D) for _ in range(3))
    q = q[:rows]
    first = 230 - rows - 20  # rows at 230 - rows .. 229, each over its last 20
    for x in ((k,) if bad == "k" else (v,) if bad == "v" else (k, v)):
        x[first - 3, 0, 4], x[first, 1, 100], x[230, 0, 3], x[240, 1, 0] = \
            float("inf"), float("nan"), float("-inf"), float("nan")
    cache.append(0, 1, k.cuda(), v.cuda())
    out = torch.full_like(q, 1.0).cuda()
    cache.window_attention(q.cuda(), out, ws.window_spec(0, 20, 2, q_start=230 - rows, kinds=(1,)), ws.WS_APPEND_RAW)
    see = ref.window_mask(n, 230 - rows, rows, 20, 2, True)
    assert not see[:, first].any() and not see[:, 230].any()
    clean = [torch.nan_to_num(x.double(), 0, 0, 0) for x in (k, v)]
    ref.check(out, *ref.attend(q.double(), *clean, see))
    # one that some rows see: theirs alone
    v[225, 0, 7] = float("inf")
    cache.append(0, 1, k.cuda(), v.cuda())
    cache.window_attention(q.cuda(), out, ws.window_spec(0, 20, 2, q_start=230 - rows, kinds=(1,)), ws.WS_APPEND_RAW)
    sees = see[:, 225]
    want, bound = ref.attend(q.double(), *clean, see)
    keep = torch.ones(rows, H, D, dtype=torch.bool)
    keep[sees, 0, 7] = False
    got = out.cpu().double()
    assert torch.isinf(got[sees, 0, 7]).all() and torch.isfinite(got[keep]).all()
    assert ((got - want).abs()[keep] <= bound[keep]).all()
    cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,rows,window,sinks,causal", [
    (12, 4096, 700, 64, True),   # a workgroup per tile and head
    (40, 920, 3000, 256, False),
    (3, 1500, 0, 0, True),       # classes, heads cut by the shares
    (12, 1000, 4000, 300, True),
    (1, 4096, 100, 0, True),
])
def test_many_tiles(ws, fmt, heads, rows, window, sinks, causal):
    """Long runs of rows over long timelines, against 64 bits on some rows; the same
    bits again, and independent of the other rows' number up to key ranges."""
    st = Stream8(ws, fmt, heads, 256, 6, 920, 0, seed=heads, max_q=4096)
    k, v = st.keys(5, (0, 1))
    n = k.shape[0]
    q = ref.normal(st.gen, rows, heads, D)
    spec = ws.window_spec(5, window, sinks, causal=causal)
    out = run(ws, st, q, spec)
    some = torch.cat([torch.tensor([0, 1, rows - 1]), torch.randperm(rows, generator=st.gen)[:24]])
    see = ref.window_mask(n, n - rows, rows, window, sinks, causal)[some]
    ref.check(out[some.cuda()], *ref.attend(q[some].double(), k, v, see))
    assert torch.equal(run(ws, st, q, spec), out)
    part = run(ws, st, q[100:700], ws.window_spec(5, window, sinks, causal=causal, q_start=n - rows + 100))
    # two results of the device, each within a few roundings of the exact one
    assert (part.float() - out[100:700].float()).norm() <= 2 * ref.U * part.float().norm()
    st.cache.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_long_timelines(ws, fmt):
    """More pages than travel in the kernel arguments (uploaded), many short pages;
    such a call is refused in a capture, a short one replays."""
    st = Stream8(ws, fmt, 1, 0, 430, 0, 4, seed=1)
    k, v = st.keys(429, (2,))
    n = k.shape[0]
    for rows, window, sinks in ((4, 1650, 16), (70, 0, 0), (4, 300, 90)):
        q = ref.normal(st.gen, rows, 1, D)
        for _ in range(2):
            out = run(ws, st, q, ws.window_spec(429, window, sinks, kinds=(2,)))
            ref.check(out, *ref.attend(q.double(), k, v, ref.window_mask(n, n - rows, rows, window, sinks, True)))
    long_call = (q.cuda(), torch.empty_like(out), ws.window_spec(429, 0, 0, kinds=(2,)), ws.WS_APPEND_RAW)
    short = (q.cuda(), torch.empty_like(out), ws.window_spec(429, 300, 90, kinds=(2,)), ws.WS_APPEND_RAW)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ws.WsError) as e:
            st.cache.window_attention(*long_call)
        st.cache.window_attention(*short)
    assert e.value.status == ws.WS_ERR_UNSUPPORTED
    for _ in range(3):
        short[1].fill_(float("nan"))
        st.cache.window_attention(*long_call)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(short[1], out)
    st.cache.close()


def test_refusals(ws):
    st = Stream8(ws, "bf16", 2, 10, 1, 20, 0)
    q = torch.zeros(4, 2, D, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 5.0)
    for kw in (dict(window=-1), dict(window=3, n_sink=-1), dict(window=3, causal=2), dict(window=3, q_start=-2),
               dict(window=3, q_start=2 ** 24 + 1)):
        spec = ws.window_spec(0, **kw)
        spec.causal = kw.get("causal", 1)
        with pytest.raises(ws.WsError) as e:
            st.cache.window_attention(q, out, spec, ws.WS_APPEND_RAW)
        assert e.value.status == ws.WS_ERR_INVALID_ARG, kw
    with pytest.raises(ws.WsError) as e:
        st.cache.window_attention(torch.zeros(1025, 2, D, dtype=torch.bfloat16, device="cuda"),
                                  torch.zeros(1025, 2, D, dtype=torch.bfloat16, device="cuda"),
                                  ws.window_spec(0, 3), ws.WS_APPEND_RAW)
    assert e.value.status == ws.WS_ERR_SHAPE
    with pytest.raises(ws.WsError):
        st.cache.window_attention(q, out, ws.window_spec(0, 3))  # positions and gamma missing
    torch.cuda.synchronize()
    assert (out == 5).all()
    st.cache.close()
