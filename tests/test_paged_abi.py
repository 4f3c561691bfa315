"""The paged cache's entry points (include/lg_paged.h) on the host: exported symbols, argument checks
(nothing is enqueued, so these run without a GPU), workspace sizes and rotary frequencies."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _lg():
    from paper_2604_10044_amd import lg
    return lg


def _map(lg, **kw):
    d = dict(batch=4, max_pages=8, n_pages=64, page_size=16, table=0x1000, pos=0x2000, len=0x3000, ref=0x4000)
    d.update(kw)
    return lg.PageMap(**d)


def _layer(lg, **kw):
    d = dict(n_pages=64, page_size=16, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=lg.LG_BF16, k=0x10000, v=0x20000)
    d.update(kw)
    return lg.PagedLayer(**d)


def test_exports_every_declared_symbol():
    lg = _lg()
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lg_paged.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(lg_[a-z_0-9]+)\s*\(", src)))
    assert len(names) == 8
    out = subprocess.run(["nm", "-D", "--defined-only", lg.LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = set(re.findall(r"\s[TW]\s+(lg_\w+)", out))
    assert not [n for n in names if n not in exported]
    assert all(hasattr(lg._lib, n) for n in names)


def test_header_compiles_as_c99(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "lg_paged.h"\nint main(void) { lg_page_map m; lg_paged_layer l; lg_rope_params p;\n'
                   'return (int)(sizeof m + sizeof l + sizeof p) == 0; }\n')
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I",
                        os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", "-c", str(src), "-o",
                        str(tmp_path / "t.o")], capture_output=True, text=True, timeout=120)
    errors = [x for x in r.stderr.splitlines() if "lg_paged.h" in x or "lg.h" in x]
    assert not errors, errors


BAD_MAPS = [(dict(table=None), 1), (dict(pos=None), 1), (dict(len=None), 1), (dict(ref=None), 1), (dict(ref=0x4004), 7),
            (dict(batch=0), 2), (dict(batch=65536), 2), (dict(max_pages=0), 2), (dict(n_pages=0), 2),
            (dict(n_pages=(1 << 28) + 1), 2), (dict(page_size=8), 3), (dict(page_size=48), 3), (dict(page_size=512), 3),
            (dict(max_pages=1 << 27), 2), (dict(batch=65535, max_pages=32769), 2)]
BAD_LAYERS = [(dict(k=None), 1), (dict(v=None), 1), (dict(k=0x10008), 7), (dict(n_pages=63), 2), (dict(page_size=32), 2),
              (dict(n_q_heads=0), 2), (dict(n_q_heads=7), 2), (dict(n_kv_heads=0), 2), (dict(n_q_heads=34), 3),
              (dict(head_dim=96), 3), (dict(dtype=2), 3)]


def _reserve(lg, m, layers=(), ws=0x50000, size=1 << 30, **kw):
    a = dict(q_start=0x10, t=0x20, base=0x30)
    a.update(kw)
    arr = (lg.PagedLayer * len(layers))(*layers) if layers else None
    return lg._lib.lg_page_reserve(ctypes.byref(m), len(layers), arr, a["q_start"], a["t"], a["base"], ws, size, None)


def _compact(lg, m, layers=(), ws=0x50000, size=1 << 30, **kw):
    a = dict(keep=0x10, nl=0x20, moved=0x30)
    a.update(kw)
    arr = (lg.PagedLayer * len(layers))(*layers) if layers else None
    return lg._lib.lg_page_compact(ctypes.byref(m), len(layers), arr, a["keep"], a["nl"], a["moved"], ws, size, None)


def _fork(lg, m, parent=0x10, ws=0x50000, size=1 << 30):
    return lg._lib.lg_page_fork(ctypes.byref(m), parent, ws, size, None)


def _attend(lg, l, m, total=8, chunk=4, window=0, sinks=0, size=1 << 34, **kw):
    a = dict(q=0x10, out=0x20, q_start=0x30, base=0x40, sw=0x50, lse=0x60, sm=0x70, conf=0x80, ws=0x90)
    a.update(kw)
    return lg._lib.lg_paged_attend(ctypes.byref(l), ctypes.byref(m), a["q"], a["out"], a["q_start"], a["base"], total,
                                   chunk, window, sinks, a["sw"], a["lse"], a["sm"], a["conf"], a["ws"], size, None)


def _rope(lg, l, m, total=8, rot=128, qs=1024, ks=256, vs=256, **kw):
    a = dict(q=0x10, k=0x20, v=0x30, freq=0x40, out=0x50, q_start=0x60, base=0x70)
    a.update(kw)
    return lg._lib.lg_rope_append(ctypes.byref(l), ctypes.byref(m), a["q"], qs, a["k"], ks, a["v"], vs, a["freq"], rot, 0,
                                  1.0, a["out"], a["q_start"], a["base"], total, None)


@pytest.mark.parametrize("bad,status", BAD_MAPS)
def test_every_call_checks_the_map(bad, status):
    lg = _lg()
    m, l = _map(lg, **bad), _layer(lg)
    assert _reserve(lg, m) == status
    assert _fork(lg, m) == status
    assert _compact(lg, m) == status
    assert _attend(lg, l, m) == status
    assert _rope(lg, l, m) == status
    assert lg.lg_page_workspace(m) == 0
    assert lg.lg_paged_attend_workspace(l, m, 8, 4) == 0


@pytest.mark.parametrize("bad,status", BAD_LAYERS)
def test_every_call_checks_the_layer(bad, status):
    lg = _lg()
    m, l = _map(lg), _layer(lg, **bad)
    assert _reserve(lg, m, [l]) == status
    assert _compact(lg, m, [_layer(lg), l]) == status
    assert _attend(lg, l, m) == status
    assert _rope(lg, l, m) == status
    assert lg.lg_paged_attend_workspace(l, m, 8, 4) == 0


def test_page_calls_reject_bad_arguments():
    lg = _lg()
    m, l = _map(lg), _layer(lg)
    need = lg.lg_page_workspace(m)
    assert need >= 4 * (4 * 8 + 4 * 8 * 16) and need % 16 == 0
    for f, names in ((_reserve, ("q_start", "t", "base")), (_compact, ("keep", "nl", "moved"))):
        for n in names:
            assert f(lg, m, **{n: None}) == 1, n
        assert f(lg, m, ws=None) == 1
        assert f(lg, m, ws=0x50008) == 7
        assert f(lg, m, size=need - 1) == 5
        assert f(lg, m, [l, _layer(lg, head_dim=64)]) == 2
        assert f(lg, m, [l, _layer(lg, dtype=lg.LG_F32)]) == 2
        assert f(lg, m, [l, _layer(lg, n_q_heads=4, n_kv_heads=4)]) == 2
    assert _fork(lg, m, parent=None) == 1
    assert _fork(lg, m, ws=None) == 1
    assert _fork(lg, m, ws=0x50004) == 7
    assert _fork(lg, m, size=need - 1) == 5
    assert lg._lib.lg_page_reserve(ctypes.byref(m), -1, None, 0x10, 0x20, 0x30, 0x50000, need, None) == 2
    assert lg._lib.lg_page_reserve(ctypes.byref(m), 1, None, 0x10, 0x20, 0x30, 0x50000, need, None) == 1
    assert lg._lib.lg_page_fork(None, 0x10, 0x50000, need, None) == 1


def test_attend_rejects_bad_arguments():
    lg = _lg()
    m, l = _map(lg), _layer(lg)
    for n in ("q", "out", "q_start", "base", "lse", "ws"):
        assert _attend(lg, l, m, **{n: None}) == 1, n
    assert _attend(lg, l, m, sw=None) == 1  # a suffix mass without a suffix
    assert _attend(lg, l, m, sw=None, sm=None) == 1
    assert _attend(lg, l, m, window=-1) == 4
    assert _attend(lg, l, m, sinks=-1) == 4
    assert _attend(lg, l, m, total=-1) == 2
    assert _attend(lg, l, m, chunk=-1) == 2
    assert _attend(lg, l, m, total=1 << 28) == 2  # 2^31 rows
    assert _attend(lg, l, m, q=0x18) == 7
    assert _attend(lg, l, m, out=0x28) == 7
    assert _attend(lg, l, m, ws=0x98) == 7
    big = _map(lg, max_pages=512)
    assert _attend(lg, l, big, size=16) == 5
    assert _attend(lg, l, m, total=0) == 0  # nothing to do, nothing enqueued
    wide = _layer(lg, n_q_heads=65535, n_kv_heads=65535)
    assert _attend(lg, wide, _map(lg, batch=65535), total=8) == 2  # more workgroups than a grid holds


def test_rope_rejects_bad_arguments():
    lg = _lg()
    m, l = _map(lg), _layer(lg)
    for n in ("q", "k", "v", "freq", "out", "q_start", "base"):
        assert _rope(lg, l, m, **{n: None}) == 1, n
    for rot in (-2, 1, 127, 130):
        assert _rope(lg, l, m, rot=rot) == 4
    assert _rope(lg, l, m, qs=1023) == 2
    assert _rope(lg, l, m, ks=255) == 2
    assert _rope(lg, l, m, vs=128) == 2
    assert _rope(lg, l, m, qs=1025) == 7
    assert _rope(lg, l, m, ks=260) == 7
    assert _rope(lg, l, m, total=-1) == 2
    assert _rope(lg, l, m, total=(1 << 23) + 1) == 2
    assert _rope(lg, l, m, q=0x18) == 7
    assert _rope(lg, l, m, v=0x38) == 7
    assert _rope(lg, l, m, out=0x58) == 7
    assert _rope(lg, l, m, total=0) == 0


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (28, 4, 128), (32, 8, 128), (16, 1, 64)])
@pytest.mark.parametrize("batch,cap", [(1, 256), (1, 16384), (7, 2048), (64, 8192)])
def test_attend_workspace_serves_smaller_steps(hq, hkv, d, batch, cap):
    """The size for a step serves every step of no more tokens and no longer chunks."""
    lg = _lg()
    m = _map(lg, batch=batch, max_pages=cap // 16)
    l = _layer(lg, n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
    most = 0
    for total in [1, 2, 3, 7, 8, 9, 31, 33, 64, 100, 127, 128, 129, 500, 1000, 1024, 4096]:
        size = lg.lg_paged_attend_workspace(l, m, total, total)
        assert size >= max(16, most), total
        most = size
        for t in {x for x in (1, 2, total // 3, total // 2, total - 1, total) if 1 <= x <= total}:
            for chunk in {1, 2, t // 2 + 1, total}:
                assert lg.lg_paged_attend_workspace(l, m, t, min(chunk, total)) <= size, (total, t, chunk)


def _params(lg, kind, **kw):
    d = dict(kind=kind, rot_dim=64, theta=1e4, factor=4.0, original_context=4096.0, slow=1.0, fast=32.0)
    d.update(kw)
    return lg.RopeParams(**d)


@pytest.mark.parametrize("rot", [2, 4, 24, 64, 128])
@pytest.mark.parametrize("kind", range(5))
def test_rope_frequencies(kind, rot):
    lg = _lg()
    p = _params(lg, kind, rot_dim=rot)
    if kind == lg.LG_ROPE_BASE and rot < 4:
        with pytest.raises(lg.LGError):
            lg.lg_rope_frequencies(p)
        return
    inv, scale = lg.lg_rope_frequencies(p)
    plain = [1e4 ** (-2 * i / rot) for i in range(rot // 2)]
    turns = [4096 * f / (2 * math.pi) for f in plain]
    assert inv.numel() == rot // 2
    assert abs(scale - (1 + 0.1 * math.log(4) if kind == lg.LG_ROPE_RAMP else 1)) < 1e-6
    for i, f in enumerate(plain):
        x = float(inv[i])
        if kind == lg.LG_ROPE_PLAIN:
            want = f
        elif kind == lg.LG_ROPE_LINEAR:
            want = f / 4
        elif kind == lg.LG_ROPE_BASE:
            want = f * 4 ** (-2 * i / (rot - 2))
        elif kind == lg.LG_ROPE_BANDS:
            want = f if turns[i] >= 32 else f / 4 if turns[i] <= 1 else \
                f * ((turns[i] - 1) / 31 + (32 - turns[i]) / 31 / 4)
        else:  # the ramp's ends are whole indices around the two borders
            at = lambda n: rot * math.log(4096 / (2 * math.pi * n)) / (2 * math.log(1e4))  # noqa: E731
            lo, hi = max(0, math.floor(at(32))), min(rot - 1, math.ceil(at(1)))
            r = min(1, max(0, (i - lo) / max(hi - lo, 1e-3)))
            want = f * (1 - r) + f / 4 * r
        assert abs(x - want) <= 2 ** -24 * want * 1.01, (i, x, want)


def test_rope_frequencies_reject():
    lg = _lg()
    f = lg._lib.lg_rope_frequencies
    s, x = ctypes.c_float(), (ctypes.c_float * 64)()
    for kind, bad in [(5, {}), (-1, {}), (0, dict(rot_dim=0)), (0, dict(rot_dim=3)), (0, dict(rot_dim=130)),
                      (0, dict(theta=1.0)), (0, dict(theta=float("nan"))), (0, dict(theta=float("inf"))),
                      (1, dict(factor=0.5)), (1, dict(factor=float("nan"))), (2, dict(rot_dim=2)),
                      (3, dict(original_context=0.0)), (3, dict(slow=0.0)), (4, dict(slow=32.0)),
                      (4, dict(fast=float("inf")))]:
        assert f(ctypes.byref(_params(lg, kind, **bad)), x, ctypes.byref(s)) == 4, (kind, bad)
    assert f(None, x, ctypes.byref(s)) == 1
    assert f(ctypes.byref(_params(lg, 0)), None, ctypes.byref(s)) == 1
    assert f(ctypes.byref(_params(lg, 0)), x, None) == 1


def test_binding_refuses_host_tensors():
    """The views take device tensors of the right types only."""
    lg = _lg()
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(lg.LGError):
        lg.page_map(i(2, 4), i(2, 64), i(2), i(16), 16)
    with pytest.raises(lg.LGError):
        lg.paged_layer(torch.zeros(16, 2, 16, 64), torch.zeros(16, 2, 16, 64), 4)
    with pytest.raises(lg.LGError):
        lg.paged_layer(torch.zeros(16, 2, 16, 64, dtype=torch.float16), torch.zeros(16, 2, 16, 64, dtype=torch.float16), 4)


def test_calls_in_place():
    """Queries may be rotated in place when their rows are dense; attention has no form in place."""
    lg = _lg()
    m, l = _map(lg), _layer(lg)
    assert _rope(lg, l, m, out=0x10, qs=1032) == 4
    assert _rope(lg, l, m, out=0x10, qs=1032, total=0) == 0
    assert _attend(lg, l, m, out=0x10) == 4
