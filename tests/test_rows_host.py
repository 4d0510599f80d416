"""Refusals of the C entries of embedding, norms of queries and keys, and dropout, without a GPU: what is wrong is reported before
anything is launched.  Addresses are never read."""
import ctypes as C

import pytest

hch = pytest.importorskip("paper_1803_11385_amd")

P = 4096          # an address, aligned to anything asked for
NAN, INF = float("nan"), float("inf")


def _sections(s):
    return None if s is None else (C.c_int32 * 3)(*s)


def _qk_fwd(t=0, X=P, lx=128, u=0, Y=2 * P, ly=128, co=P, n=4, h=4, hq=2, hk=1, d=32, s=(4, 4, 4), base=1e4, scale=1.0, eps=1e-5):
    return hch.load_library().hch_qknorm_rope_fwd(t, X, lx, u, Y, ly, None, None, co, n, h, hq, hk, d, _sections(s), base, scale, eps, None)


def _qk_bwd(t=0, X=P, lx=128, u=0, dY=2 * P, ly=128, v=0, dX=3 * P, lz=128, dq=P, dk=P, co=P, n=4, h=4, hq=2, hk=1, d=32, s=(4, 4, 4), base=1e4,
            scale=1.0, eps=1e-5, ws=P, nb=1 << 20):
    return hch.load_library().hch_qknorm_rope_bwd(t, X, lx, u, dY, ly, v, dX, lz, None, None, dq, dk, co, n, h, hq, hk, d, _sections(s), base,
                                                  scale, eps, ws, nb, None)


def test_qknorm_refuses():
    for f in (_qk_fwd, _qk_bwd):
        assert f(t=2) == 1 and f(u=-1) == 1 and f(X=None) == 1 and f(co=None) == 1 and f(s=None) == 1
        assert f(n=-1) == 1 and f(h=0) == 1 and f(hq=-1) == 1 and f(hk=-1) == 1 and f(hq=3, hk=2) == 1 and f(d=31) == 1 and f(d=0) == 1
        assert f(hq=2 ** 31 - 1, hk=2 ** 31 - 1) == 1
        assert f(lx=127) == 1 and f(ly=127) == 1 and f(s=(16, 1, 0)) == 1 and f(s=(-1, 0, 0)) == 1 and f(s=(2 ** 31 - 1,) * 3) == 1
        assert f(base=0.0) == 1 and f(base=INF) == 1 and f(scale=NAN) == 1 and f(eps=-1.0) == 1 and f(eps=NAN) == 1 and f(eps=INF) == 1
        assert f(d=258, lx=2000, ly=2000) == 5 and f(h=1 << 24, d=256, lx=1 << 33, ly=1 << 33) == 5
        assert f(h=2 ** 31 - 1, d=256, lx=1 << 50, ly=1 << 50) == 5
    assert _qk_fwd(Y=None) == 1 and _qk_fwd(Y=P, u=1) == 1 and _qk_fwd(Y=P, ly=256) == 1
    assert _qk_bwd(dY=None) == 1 and _qk_bwd(dX=None) == 1 and _qk_bwd(v=7) == 1 and _qk_bwd(lz=127) == 1
    assert _qk_bwd(dX=2 * P, v=1) == 1 and _qk_bwd(dX=2 * P, lz=256) == 1 and _qk_bwd(dX=P, v=1) == 1 and _qk_bwd(dX=P, lz=256) == 1
    assert _qk_bwd(dq=None) == 1 and _qk_bwd(dk=None) == 1
    assert _qk_bwd(ws=None) == 1 and _qk_bwd(ws=P + 128) == 1 and _qk_bwd(nb=255) == 6
    assert b"hch_qknorm_rope_bwd" in hch.load_library().hch_last_error()
    # 2^24 workgroups of 256 cannot be started: a row of 1024 lanes or more has a workgroup to itself
    assert _qk_fwd(n=1 << 28, h=1 << 14, d=256, hq=1, hk=1, lx=1 << 22, ly=1 << 22) == 5


def test_qknorm_nothing_to_do():
    assert _qk_fwd(n=0, X=None, Y=None, co=None) == 0
    assert _qk_fwd(Y=P, hq=0, hk=0, co=None) == 0                    # in place without a head to turn
    assert _qk_bwd(n=0, X=None, dY=None, dX=None, co=None, dq=None, dk=None, ws=None, nb=0) == 0
    assert _qk_fwd(n=0, d=31) == 1 and _qk_bwd(n=0, eps=NAN) == 1


def test_qknorm_workspace():
    ask = hch.hch_qknorm_rope_workspace_bytes
    assert ask(0, 1, 1, 64) == 256 and ask(1, 1, 1, 64) >= 2 * 64 * 4 and ask(10 ** 9, 8, 8, 256) <= 1 << 23
    assert ask(-1, 1, 1, 64) == 0 and ask(1, -1, 1, 64) == 0 and ask(1, 1, -1, 64) == 0 and ask(1, 1, 1, 63) == 0 and ask(1, 1, 1, 258) == 0


def _drop(t=0, X=P, R=None, u=0, Y=2 * P, n=4, c=8, p=0.1, seed=0, step=None):
    return hch.load_library().hch_dropout_fwd(t, X, R, u, Y, n, c, p, seed, step, None)


def _drop_bwd(t=0, X=P, u=0, Y=2 * P, n=4, c=8, p=0.1, seed=0, step=None):
    return hch.load_library().hch_dropout_bwd(t, X, u, Y, n, c, p, seed, step, None)


def _norm_fwd(t=0, X=P, R=2 * P, S=3 * P, u=0, Y=4 * P, n=4, c=8, eps=1e-5, p=0.1, step=None):
    return hch.load_library().hch_dropout_layernorm_fwd(t, X, R, S, None, None, u, Y, None, n, c, eps, p, 0, step, None)


def _norm_bwd(t=0, X=P, st=P, u=0, Y=2 * P, dR=3 * P, v=0, dX=4 * P, dg=P, db=P, n=4, c=8, p=0.1, step=None, ws=P, nb=1 << 20):
    return hch.load_library().hch_dropout_layernorm_bwd(t, X, st, None, u, Y, None, dR, v, dX, dg, db, n, c, p, 0, step, ws, nb, None)


def test_dropout_refuses():
    for f in (_drop, _drop_bwd, _norm_fwd, _norm_bwd):
        assert f(t=2) == 1 and f(u=-1) == 1 and f(X=None) == 1 and f(Y=None) == 1 and f(n=-1) == 1 and f(c=0) == 1 and f(c=-8) == 1
        assert f(p=-0.1) == 1 and f(p=1.1) == 1 and f(p=NAN) == 1 and f(p=INF) == 1 and f(step=P + 4) == 1
    for f in (_drop, _drop_bwd):
        assert f(Y=P, u=1) == 1 and f(n=1 << 62) == 5 and f(n=1 << 40, c=1 << 21) == 5 and f(n=0, X=None, Y=None) == 0 and f(n=0, p=2.0) == 1
    assert b"hch_dropout_bwd" in hch.load_library().hch_last_error()
    assert _norm_fwd(R=None) == 1 and _norm_fwd(S=None) == 1 and _norm_fwd(eps=-1.0) == 1 and _norm_fwd(eps=NAN) == 1 and _norm_fwd(c=8193) == 5
    assert _norm_fwd(n=0, X=None, R=None, S=None, Y=None) == 0
    assert _norm_bwd(st=None) == 1 and _norm_bwd(dR=None) == 1 and _norm_bwd(dX=None) == 1 and _norm_bwd(dX=3 * P) == 1 and _norm_bwd(v=5) == 1
    assert _norm_bwd(dg=None) == 1 and _norm_bwd(db=None) == 1 and _norm_bwd(c=8193) == 5
    assert _norm_bwd(ws=None) == 1 and _norm_bwd(ws=P + 8) == 1 and _norm_bwd(nb=64) == 6
    assert _norm_bwd(n=0, X=None, st=None, Y=None, dR=None, dX=None, dg=None, db=None, ws=None, nb=0) == 0


def test_dropout_with_norm_refuses_tensors_that_overwrite_each_other():
    """Rows of one type in place of rows of another are written over rows that other workgroups have still to read; Y in S's place, and dX in
    that of any other tensor, leave one result where two are promised."""
    def bwd(t=0, S=P, u=0, dY=2 * P, dS=None, dR=3 * P, v=0, dX=4 * P, n=4):
        return hch.load_library().hch_dropout_layernorm_bwd(t, S, P, None, u, dY, dS, dR, v, dX, None, None, n, 8, 0.1, 0, None, None, 0, None)

    for t, u in ((0, 1), (1, 0)):
        assert _norm_fwd(t=t, u=u, Y=P) == 1 and _norm_fwd(t=t, u=u, Y=2 * P) == 1 and _norm_fwd(t=t, u=u, Y=3 * P) == 1
        assert bwd(t=t, u=u, dR=2 * P) == 1
    for t in (0, 1):
        assert _norm_fwd(t=t, u=t, Y=3 * P) == 1 and _norm_fwd(t=t, u=t, S=P, Y=P) == 1 and _norm_fwd(t=t, u=t, S=2 * P, Y=2 * P) == 1
        for v in (0, 1):
            assert bwd(t=t, v=v, dX=P) == 1 and bwd(t=t, u=v, v=v, dX=2 * P) == 1 and bwd(t=t, v=v, dS=5 * P, dX=5 * P) == 1
            assert bwd(t=t, v=v, dX=3 * P) == 1
    assert b"hch_dropout_layernorm_bwd" in hch.load_library().hch_last_error()
    assert bwd(n=0, S=None, dY=None, dR=None, dX=None) == 0 and bwd(n=0, S=P, dY=P, dR=P, dX=P) == 0
    assert _norm_fwd(n=0, X=P, R=P, S=P, Y=P, u=1) == 0


def _embed(t=0, T=P, ids=P, u=0, Y=P, ld=8, n=4, c=8, vocab=10, scale=1.0):
    return hch.load_library().hch_embed_fwd(t, T, ids, u, Y, ld, n, c, vocab, scale, None)


def _embed_bwd(ids=P, t=0, dY=P, ld=8, dT=P, n=4, c=8, vocab=10, scale=1.0, ws=P, nb=1 << 62):
    return hch.load_library().hch_embed_bwd(ids, t, dY, ld, dT, n, c, vocab, scale, ws, nb, None)


def test_embedding_refuses():
    for f in (_embed, _embed_bwd):
        assert f(t=2) == 1 and f(ids=None) == 1 and f(n=-1) == 1 and f(c=0) == 1 and f(vocab=0) == 1 and f(vocab=-5) == 1
        assert f(scale=NAN) == 1 and f(scale=INF) == 1 and f(ld=7) == 1
        assert f(n=1 << 31) == 5 and f(n=(1 << 31) - 4095) == 5 and f(c=(1 << 22) + 1, ld=1 << 23) == 5
    assert _embed(u=2) == 1 and _embed(T=None) == 1 and _embed(Y=None) == 1 and _embed(n=0, T=None, ids=None, Y=None) == 0
    assert _embed_bwd(dY=None) == 1 and _embed_bwd(dT=None) == 1 and _embed_bwd(n=0, dT=None) == 1
    assert _embed_bwd(ws=None) == 1 and _embed_bwd(ws=P + 64) == 1 and _embed_bwd(nb=255) == 6
    assert b"hch_embed_bwd" in hch.load_library().hch_last_error()
    # 2^24 workgroups cannot be started: one for each 64 rows where rows are wide
    assert _embed_bwd(c=4096, ld=4096, n=(1 << 30) + 1) == 5


def test_embedding_workspace():
    ask = hch.hch_embed_workspace_bytes
    assert ask(0, 8, 10) == 256 and ask(-1, 8, 10) == 0 and ask(1, 0, 10) == 0 and ask(1, 8, 0) == 0 and ask(1 << 31, 8, 10) == 0
    for n, c, vocab in ((1, 1, 1), (64, 3, 7), (100000, 64, 50), (5, 8, 10 ** 6)):
        assert ask(n, c, vocab) % 256 == 0 and ask(n, c, vocab) >= 16 * n + 4 * vocab + (n + 1023) // 1024 * 2 * c * 4


def test_binding_refuses_before_the_library_is_reached():
    import torch
    t = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: hch.hch_dropout_fwd(hch.HCH_F32, t, None, hch.HCH_F32, t, 4, 8, 0.1, 0),
                 lambda: hch.hch_embed_fwd(hch.HCH_F32, t, ids, hch.HCH_F32, t, 4, 8, 4),
                 lambda: hch.hch_qknorm_rope_fwd(hch.HCH_F32, t, hch.HCH_F32, t, None, None, None, 4, 1, 1, 0, 8, (0, 0, 0))):
        with pytest.raises(hch.HchError, match="GPU memory"):
            call()
    with pytest.raises(hch.HchError, match="seed"):
        hch.hch_dropout_bwd(hch.HCH_F32, None, hch.HCH_F32, None, 0, 8, 0.1, -1)
    with pytest.raises(hch.HchError, match="out of range"):
        hch.hch_embed_bwd(None, hch.HCH_F32, None, None, 0, 1 << 32, 5, 1.0, None)


def test_tensors_of_another_gpu_are_refused(monkeypatch):
    """The calls run on the current device: an address of another one's memory would be read there."""
    import torch
    from paper_1803_11385_amd import binding

    class There:
        def __init__(self, device):
            self.device_index = device

        def get_device(self):
            return self.device_index

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    assert binding._on(77, There(1), None, There(1)) == 77
    with pytest.raises(hch.HchError, match="GPU 0"):
        binding._on(77, There(1), There(0))


def test_embedding_refuses_rows_of_other_types():
    """Rows of fp16 or of integers are as wide as rows of bf16: their bits would be taken for bf16's."""
    import torch
    from paper_1803_11385_amd import pipeline
    emb = pipeline.Embedding(4, 9, 8, device="cpu")
    for call in (emb.forward, emb.backward):
        for t in (torch.float16, torch.int16, torch.uint8, torch.float64):
            with pytest.raises(hch.HchError, match=f"element type {t}"):
                call(torch.zeros((4, 8), dtype=t))
        for t in (torch.float32, torch.bfloat16):               # goes on to where the tensor's place is looked at
            with pytest.raises(hch.HchError, match="GPU memory"):
                call(torch.zeros((4, 8), dtype=t))


def test_a_block_with_dropout_needs_a_seed():
    """Blocks with one seed drop the same elements in every step: none is taken that the program did not choose."""
    from paper_1803_11385_amd import pipeline

    class Reached(Exception):
        pass

    class Levels:
        def n(self, level):
            raise Reached

    for p in (0.1, 0.0):
        with pytest.raises(hch.HchError, match="seed"):
            pipeline.AttentionBlock(Levels(), 0, 32, 2, 2, 16, dropout=p)
        for seed in (-1, 2 ** 64):
            with pytest.raises(hch.HchError, match="seed"):
                pipeline.AttentionBlock(Levels(), 0, 32, 2, 2, 16, dropout=p, seed=seed)
        for seed in (0, 2 ** 64 - 1):
            with pytest.raises(Reached):
                pipeline.AttentionBlock(Levels(), 0, 32, 2, 2, 16, dropout=p, seed=seed)
    with pytest.raises(Reached):
        pipeline.AttentionBlock(Levels(), 0, 32, 2, 2, 16)
