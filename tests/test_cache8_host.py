"""Host side of the 8-bit cache and the token window, without a GPU: refusals that
come before any device call, struct layouts, the order of a window's timeline."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2607_04443_amd import _build
    if not (os.path.exists(_build.LIB_PATH) and os.path.exists(_build.HOST_LIB_PATH)):
        _build.build()
    return ctypes.CDLL(_build.LIB_PATH), ctypes.CDLL(_build.HOST_LIB_PATH)


def test_refusals_before_any_device_call(lib):
    from paper_2607_04443_amd import ws
    cfg = ws.ws_cache_config()
    for fmt in (-1, 3, 100):
        with pytest.raises(ws.WsError) as e:
            ws.ws_cache_create_format(cfg, fmt)
        assert e.value.status == ws.WS_ERR_INVALID_ARG and "format" in str(e.value)
    with pytest.raises(ValueError):
        ws.Cache(2, 4, kv_format="fp8")
    ws_lib = lib[0]
    for name, args in (("ws_cache_format", [None, None]), ("ws_kv_gather", [None, 1, None, None]),
                       ("ws_cache_export_codes", [None, 0, 0, None, None, None, None]),
                       ("ws_cache_create_format", [None, 1, None])):
        assert getattr(ws_lib, name)(*args) == ws.WS_ERR_INVALID_ARG, name
    null, i64 = ctypes.c_void_p(), ctypes.c_int64
    f = ws_lib.ws_window_attention
    spec, desc = ws.window_spec(0, 3), ws.ws_query_desc()
    assert f(null, i64(0), i64(0), 1, ctypes.byref(desc), null, None, null, i64(0), i64(0), null) == 1
    assert f(null, i64(0), i64(0), 1, ctypes.byref(desc), null, ctypes.byref(spec), null, i64(0), i64(0), null) == 1


def test_struct_layouts(tmp_path):
    from paper_2607_04443_amd import ws
    src, exe = tmp_path / "p.c", tmp_path / "p"
    fields = {"ws_window_spec": ["mask", "window", "n_sink", "causal", "q_start"],
              "ws_gather_item": ["unit", "kind", "n_tokens", "k_out", "v_out", "tok_stride", "head_stride"]}
    body = "".join(f'printf("%zu ", sizeof({t}));' + "".join(f'printf("%zu ", offsetof({t}, {f}));' for f in fs)
                   for t, fs in fields.items())
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"ws.h\"\nint main(void) {" + body +
                   'printf("%d %d %d %d", WS_KV_BF16, WS_KV_INT8, WS_KV_E4M3, WS_WINDOW_AT_END); return 0; }')
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for t, fs in fields.items():
        c = getattr(ws, t)
        want += [ctypes.sizeof(c)] + [getattr(c, f).offset for f in fs]
    assert got == want + [ws.WS_KV_BF16, ws.WS_KV_INT8, ws.WS_KV_E4M3, ws.WS_WINDOW_AT_END]


def test_timeline_order(lib):
    """By unit, then kind, whatever the order of the appends and of the pages."""
    host = lib[1]
    host.wsh_create.restype = ctypes.c_void_p
    host.wsh_create.argtypes = [ctypes.c_int32] * 2
    host.wsh_destroy.argtypes = [ctypes.c_void_p]
    host.wsh_acquire.argtypes = [ctypes.c_void_p] + [ctypes.c_int32] * 3 + [ctypes.c_void_p]
    host.wsh_release.argtypes = [ctypes.c_void_p] + [ctypes.c_int32] * 2
    host.wsh_timeline.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_uint32,
                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p]
    host.wsh_segment_pages.argtypes = [ctypes.c_void_p] + [ctypes.c_int32] * 2 + [ctypes.c_void_p, ctypes.c_int32]
    pt = host.wsh_create(64, 40)
    created = ctypes.c_int32()
    sizes = {(2, 1): 70, (0, 1): 64, (2, 2): 3, (1, 1): 130, (0, 0): 100, (1, 2): 4, (3, 0): 20, (5, 1): 9}
    for (u, k), n in sizes.items():
        assert host.wsh_acquire(pt, u, k, n, ctypes.byref(created)) == 0
    host.wsh_release(pt, 0, 1)  # taken again, last
    assert host.wsh_acquire(pt, 0, 1, 65, ctypes.byref(created)) == 0
    sizes[0, 1] = 65

    def timeline(q_unit, min_unit, kinds):
        page, valid, n = np.zeros(64, np.int32), np.zeros(64, np.int32), ctypes.c_int64()
        m = host.wsh_timeline(pt, q_unit, min_unit, kinds, page.ctypes.data, valid.ctypes.data, 64, ctypes.byref(n))
        return list(zip(page[:m].tolist(), valid[:m].tolist())), n.value

    for q_unit, low, kinds in ((9, -5, 7), (3, -5, 7), (3, 1, 7), (2, 2, 3), (9, 0, 4), (-1, -5, 7), (9, 0, 0)):
        want, total = [], 0
        for (u, k), n in sorted(sizes.items()):
            if kinds >> k & 1 and u <= q_unit and (k == 0 or u >= low):
                ids = np.zeros(64, np.int32)
                m = host.wsh_segment_pages(pt, u, k, ids.ctypes.data, 64)
                want += [(int(ids[i]), min(64, n - 64 * i)) for i in range(m)]
                total += n
        assert timeline(q_unit, low, kinds) == (want, total)
    host.wsh_destroy(pt)
