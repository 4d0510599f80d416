"""Refusals of the attention block's C entries, without a GPU: what is wrong is reported before anything is launched.
Addresses are never read."""
import ctypes as C
import os
import subprocess
import sys

import pytest

hch = pytest.importorskip("paper_1803_11385_amd")
from paper_1803_11385_amd import binding  # noqa: E402

P = 4096          # an address, aligned to anything asked for


def _desc(**kw):
    d = dict(dtype=0, batch=1, heads_q=2, heads_kv=1, head_dim=32, scale=1.0, n_q=4, n_k=6, q_offsets=P, k_offsets=P, ld_q=64, ld_k=32,
             ld_v=32, ld_o=64, ld_do=64, ld_dq=64, ld_dk=32, ld_dv=32)
    d.update(kw)
    return binding._AttnDesc(**d)


def _fwd(ws=P, nbytes=1 << 30, q=P, o=P, **kw):
    return hch.load_library().hch_attn_fwd(C.byref(_desc(**kw)), q, P, P, o, None, ws, nbytes, None)


def _bwd(ws=P, nbytes=1 << 30, do=P, lse=P, **kw):
    return hch.load_library().hch_attn_bwd(C.byref(_desc(**kw)), P, P, P, P, lse, do, P, P, P, ws, nbytes, None)


def test_attention_refuses():
    L = hch.load_library()
    assert L.hch_attn_fwd(None, P, P, P, P, None, P, 1 << 30, None) == 1
    for f in (_fwd, _bwd):
        assert f(dtype=2) == 1 and f(heads_q=3, heads_kv=2) == 1 and f(heads_kv=0) == 1 and f(head_dim=0) == 1
        assert f(batch=-1) == 1 and f(n_q=-1) == 1 and f(batch=0) == 1
        assert f(scale=0.0) == 1 and f(scale=-1.0) == 1 and f(scale=float("nan")) == 1
        assert f(q_offsets=None) == 1 and f(k_offsets=None) == 1
        assert f(ld_q=63) == 1 and f(ld_v=31) == 1
        assert f(head_dim=129, ld_q=512, ld_o=512, ld_k=512, ld_v=512) == 5
        assert f(ld_k=1 << 22) == 5 and f(n_k=1 << 31) == 5 and f(n_q=1 << 31) == 5
        assert f(ws=None) == 1 and f(ws=P + 128) == 1 and f(nbytes=255) == 6
    assert _fwd(q=None) == 1 and _fwd(o=None) == 1
    assert _bwd(do=None) == 1 and _bwd(lse=None) == 1 and _bwd(ld_dq=63) == 1 and _bwd(ld_dv=31) == 1 and _bwd(ld_dk=1 << 22) == 5
    assert b"hch_attn_bwd" in L.hch_last_error()
    assert _fwd(n_q=0) == 0                               # nothing to do: nothing is launched
    assert _bwd(n_q=0, n_k=0) == 0 and _bwd(batch=0, n_q=0, n_k=0) == 0


def test_attention_refuses_rows_whose_last_tile_would_end_beyond_32_bits():
    last = 2 ** 31 - 257
    ask = lambda **kw: hch.load_library().hch_attn_workspace_bytes(C.byref(_desc(**kw)), hch.HCH_WS_FWD)
    assert ask(n_k=last) and not ask(n_k=last + 1)
    one = dict(heads_q=1, heads_kv=1)
    assert ask(n_q=last, **one) and not ask(n_q=last + 1, **one) and not ask(n_q=last // 2 + 1, heads_q=2, heads_kv=1)


def test_attention_workspace():
    ask = hch.hch_attn_workspace_bytes
    assert ask(hch.HCH_WS_FWD, hch.HCH_F32, 1, 0, 0, 2, 1, 32) == 256
    assert ask(hch.HCH_WS_BWD_DATA, hch.HCH_BF16, 0, 0, 0, 2, 1, 32) == 256
    assert ask(hch.HCH_WS_BWD_WEIGHT, hch.HCH_F32, 1, 4, 6, 2, 1, 32) == 0
    assert ask(hch.HCH_WS_FWD, hch.HCH_F32, 1, 4, 6, 2, 3, 32) == 0 and ask(hch.HCH_WS_FWD, hch.HCH_F32, 1, 4, 6, 2, 1, 200) == 0
    # parts of a split are fp32 rows with a maximum and a sum: bounded by 256 of them
    few = ask(hch.HCH_WS_FWD, hch.HCH_BF16, 8, 8, 609323, 8, 2, 32)
    assert 256 < few <= 256 * 8 * 8 * (32 * 4 + 8) + 512
    for d in (1, 20, 64, 128):
        for n in (1, 100, 5000):
            assert ask(hch.HCH_WS_BWD_DATA, hch.HCH_F32, 1, n, n, 2, 1, d) >= 4 * n * 2


def test_norm_refuses():
    L = hch.load_library()
    fwd = lambda t=0, X=P, R=None, S=None, u=0, Y=P, n=4, c=8, eps=1e-5: L.hch_layernorm_fwd(t, X, R, S, None, None, u, Y, None, n, c, eps, None)
    assert fwd(t=3) == 1 and fwd(u=-1) == 1 and fwd(X=None) == 1 and fwd(Y=None) == 1 and fwd(R=P) == 1 and fwd(S=P) == 1
    assert fwd(n=-1) == 1 and fwd(c=0) == 1 and fwd(eps=-1e-9) == 1 and fwd(eps=float("nan")) == 1 and fwd(c=8193) == 5
    assert fwd(n=0) == 0
    bwd = lambda t=0, X=P, st=P, u=0, dY=P, dX=P, dg=P, db=P, n=4, c=8, ws=P, nb=1 << 20: L.hch_layernorm_bwd(
        t, X, st, None, u, dY, None, dX, dg, db, n, c, ws, nb, None)
    assert bwd(t=3) == 1 and bwd(u=9) == 1 and bwd(X=None) == 1 and bwd(st=None) == 1 and bwd(dY=None) == 1 and bwd(dX=None) == 1
    assert bwd(dg=None) == 1 and bwd(db=None) == 1 and bwd(n=-1) == 1 and bwd(c=0) == 1 and bwd(c=9000) == 5
    assert bwd(ws=None) == 1 and bwd(ws=P + 16) == 1 and bwd(nb=64) == 6
    assert bwd(n=0, dg=None, db=None, ws=None, nb=0) == 0
    assert hch.hch_layernorm_workspace_bytes(1000, 64) % 256 == 0 and hch.hch_layernorm_workspace_bytes(5, 0) == 0


def test_rope_refuses():
    L = hch.load_library()

    def f(t=0, X=P, lx=64, u=0, Y=2 * P, ly=64, co=P, n=4, h=2, r=2, d=32, s=(4, 4, 4), base=1e4, scale=1.0):
        return L.hch_rope_fwd(t, X, lx, u, Y, ly, co, n, h, r, d, (C.c_int32 * 3)(*s), base, scale, None)

    assert f(t=2) == 1 and f(u=2) == 1 and f(X=None) == 1 and f(Y=None) == 1 and f(co=None) == 1
    assert f(n=-1) == 1 and f(h=0) == 1 and f(r=3) == 1 and f(r=-1) == 1 and f(d=31) == 1 and f(d=0) == 1
    assert f(lx=63) == 1 and f(ly=63) == 1 and f(s=(8, 8, 1)) == 1 and f(s=(-1, 0, 0)) == 1 and f(s=(2 ** 31 - 1, 2 ** 31 - 1, 5)) == 1
    assert f(base=0.0) == 1 and f(base=float("inf")) == 1 and f(scale=float("nan")) == 1
    assert f(Y=P, u=1) == 1 and f(Y=P, ly=128) == 1       # in place with another type, another stride
    assert f(d=258, lx=1000, ly=1000) == 5
    assert f(n=0) == 0
    assert L.hch_rope_bwd(0, P, 64, 0, P, 64, None, 4, 2, 2, 32, (C.c_int32 * 3)(1, 1, 1), 1e4, 1.0, None) == 1
    assert b"hch_rope_bwd" in L.hch_last_error()


def test_one_hip_runtime_whichever_is_imported_first():
    """torch ships a HIP runtime; with the library's loaded beside it neither would work."""
    code = ("import paper_1803_11385_amd, torch\n"
            "print(len({l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64' in l}))")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300, check=True)
    assert out.stdout.split()[-1] == "1", out.stdout


def test_rope_refuses_rows_whose_length_passes_32_bits():
    """2^24 heads of 256 channels: the product is 2^32.  In a process of its own, which has to end by itself."""
    code = ("import ctypes as C\nimport paper_1803_11385_amd as hch\n"
            "print(hch.load_library().hch_rope_fwd(0, 4096, 1 << 33, 0, 8192, 1 << 33, 4096, 4, 1 << 24, 1, 256, (C.c_int32 * 3)(1, 1, 1), 1e4, 1.0, None))")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.split()[-1] == "5", (out.returncode, out.stdout, out.stderr[-300:])


def test_no_rows_need_no_tensors():
    """The address of a tensor without elements is null: with n = 0 that is no error in any of the entries."""
    L = hch.load_library()
    assert L.hch_layernorm_fwd(0, None, None, None, None, None, 0, None, None, 0, 8, 1e-5, None) == 0
    assert L.hch_layernorm_bwd(0, None, None, None, 0, None, None, None, None, None, 0, 8, None, 0, None) == 0
    for f in (L.hch_rope_fwd, L.hch_rope_bwd):
        assert f(0, None, 64, 1, None, 64, None, 0, 2, 2, 32, (C.c_int32 * 3)(1, 1, 1), 1e4, 1.0, None) == 0
    # what does not depend on the rows is still looked at
    assert L.hch_layernorm_fwd(0, None, None, None, None, None, 0, None, None, 0, 0, 1e-5, None) == 1
    assert L.hch_layernorm_fwd(0, None, P, None, None, None, 0, None, None, 0, 8, 1e-5, None) == 1
    assert L.hch_layernorm_bwd(0, None, None, None, 0, None, None, None, P, None, 0, 8, P, 1 << 20, None) == 1
    assert L.hch_rope_fwd(0, None, 64, 1, None, 64, None, 0, 2, 2, 32, None, 1e4, 1.0, None) == 1


def test_attention_refuses_launches_of_2_to_24_workgroups():
    """A launch's work items are counted in 32 bits: 2^24 workgroups of 256 are refused before anything is launched.  (Sizes beyond
    the limit only: others would be launched.)"""
    one = dict(heads_q=1, heads_kv=1, nbytes=1 << 62)
    many = dict(heads_q=16, heads_kv=16, nbytes=1 << 62, **{ld: 512 for ld in ("ld_q", "ld_k", "ld_v", "ld_o", "ld_do", "ld_dq", "ld_dk", "ld_dv")})
    for f in (_fwd, _bwd):
        assert f(n_q=2 ** 31 - 257, n_k=1 << 20, batch=1 << 23, **one) == 5       # tiles of rows
        assert f(n_q=1 << 24, n_k=1 << 24, batch=1 << 24, **one) == 5             # shapes of one row
        assert f(n_q=1 << 20, n_k=1 << 20, batch=1 << 20, **many) == 5            # for each of 16 key heads
    assert _bwd(n_q=8, n_k=2 ** 31 - 257, batch=8, **many) == 5                   # one pass of the gradient would fit


def test_rope_refuses_launches_of_2_to_24_workgroups():
    f = hch.load_library().hch_rope_fwd
    assert f(0, P, 1 << 22, 0, 2 * P, 1 << 22, P, 1 << 28, 1 << 14, 1, 256, (C.c_int32 * 3)(1, 1, 1), 1e4, 1.0, None) == 5


def test_offsets_and_positions_of_a_level_go_where_they_are_asked_for():
    import numpy as np
    import synth_shapes as S
    coords, offs, _ = S.config_batch(2, batch=3, u=16)
    lv = hch.hch_build_tables_host(coords, offs, 16, 2)
    for level in range(2):
        o, p = lv.device_offsets(level, "cpu"), lv.device_positions(level, "cpu")
        assert o.device.type == p.device.type == "cpu"
        assert o.dtype == p.dtype and o.tolist() == lv.info(level).N.tolist() and np.array_equal(p.numpy(), lv.info(level).coords_host())
