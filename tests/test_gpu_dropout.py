"""hch_dropout_* and hch_dropout_layernorm_* against the 64-bit oracle.

Bounds: k x is off by two roundings of fp32 (the factor's and the product's), the sum by one more, a result in bf16 by half a step of
its own, 2^-8.  The norm's bounds are those of layer norm: sums over c channels off by c 2^-24 of their terms' sizes."""
import numpy as np
import pytest

from oracle import block as K
from oracle import rows as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
hch = pytest.importorskip("paper_1803_11385_amd")

TYPES = {"f32": (hch.HCH_F32, torch.float32), "bf16": (hch.HCH_BF16, torch.bfloat16)}
U = 2.0 ** -24
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}      # beyond the roundings of fp32 that are counted
ALL = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")]


def _on(rng, shape, dtype, offset=0):
    """A tensor on the GPU that begins `offset` elements behind a 256-byte border, and its values."""
    x = torch.from_numpy(rng.normal(size=shape).astype(np.float32)).to(TYPES[dtype][1])
    t = torch.zeros(x.numel() + offset, dtype=x.dtype, device="cuda")[offset:].view(shape)
    t.copy_(x)
    return t, x.double().numpy()


def _near(got, want, bound, what):
    torch.cuda.synchronize()
    off = np.abs(got.double().cpu().numpy() - want) - bound
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} of {off.size} beyond the bound, worst {off.max()}"


def _step(v):
    return torch.full((1,), v, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("x,y", ALL)
@pytest.mark.parametrize("c", [1, 2, 3, 7, 8, 9, 16, 50, 64, 100, 250, 256, 1030, 4096, 4100, 9001])
def test_dropout(x, y, c):
    rng = np.random.default_rng(c)
    for n, p, residual, offset, step in ((1, 0.5, True, 0, None), (67, 0.1, False, 0, 5), (1200 if c < 300 else 37, 0.25, True, 1, -3)):
        seed = int(rng.integers(0, 2 ** 63)) * 2 + 1
        X, xs = _on(rng, (n, c), x, offset)
        Rr, rs = _on(rng, (n, c), y, offset) if residual else (None, 0.0)
        guard = torch.full((n * c + 64,), 7.0, dtype=TYPES[y][1], device="cuda")
        Y = guard[offset: offset + n * c].view(n, c)
        at = None if step is None else _step(step)
        hch.hch_dropout_fwd(TYPES[x][0], X, Rr, TYPES[y][0], Y, n, c, p, seed, at)
        k = R.dropout_factors(n, c, p, seed, step or 0)
        want = k * xs + rs
        _near(Y, want, 2 * U * np.abs(k * xs) + U * np.abs(want) + HALF[y] * (np.abs(want) * (1 + U) + 3 * U * np.abs(k * xs)), "y")
        assert (guard[n * c + offset:] == 7).all() and (offset == 0 or guard[0] == 7)
        if not residual:
            assert ((Y == 0).cpu().numpy() == ((k == 0) | (xs == 0))).all()
        # the way back has the same mask, whatever the types
        dY, dys = _on(rng, (n, c), y, offset)
        dX = torch.full((n, c), float("nan"), dtype=TYPES[x][1], device="cuda")
        hch.hch_dropout_bwd(TYPES[y][0], dY, TYPES[x][0], dX, n, c, p, seed, at)
        _near(dX, k * dys, (2 * U + HALF[x] * (1 + 2 * U)) * np.abs(k * dys), "dx")


@pytest.mark.parametrize("c", [50, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_in_place_and_at_the_ends_of_p(dtype, c):
    rng = np.random.default_rng(3)
    code, n = TYPES[dtype][0], 333
    X, xs = _on(rng, (n, c), dtype)
    Y = torch.empty_like(X)
    hch.hch_dropout_fwd(code, X, None, code, Y, n, c, 0.0, 1)
    assert torch.equal(X, Y)
    hch.hch_dropout_fwd(code, X, None, code, Y, n, c, 1.0, 1)
    assert not Y.any()
    hch.hch_dropout_fwd(code, X, X, code, Y, n, c, 1.0, 1)                 # nothing but r
    assert torch.equal(X, Y)
    hch.hch_dropout_fwd(code, X, None, code, Y, n, c, 1.0 - 2.0 ** -16, 9)  # the last p below 1: one in 65536 is kept
    k = R.dropout_factors(n, c, 1.0 - 2.0 ** -16, 9)
    _near(Y, k * xs, (2 * U + HALF[dtype] * (1 + 2 * U)) * np.abs(k * xs), "y")
    hch.hch_dropout_fwd(code, X, None, code, Y, n, c, 0.3, 2 ** 64 - 1)
    Z = X.clone()
    hch.hch_dropout_fwd(code, Z, None, code, Z, n, c, 0.3, 2 ** 64 - 1)    # y = x
    assert torch.equal(Y, Z)
    Rr, _ = _on(rng, (n, c), dtype)
    hch.hch_dropout_fwd(code, X, Rr, code, Y, n, c, 0.3, 77)
    hch.hch_dropout_fwd(code, X, Rr, code, Rr, n, c, 0.3, 77)              # y = r
    assert torch.equal(Y, Rr)


def test_what_is_dropped_may_hold_anything():
    n, c, p = 40, 20, 0.5
    k = torch.from_numpy(R.dropout_factors(n, c, p, 11)).cuda()
    for bad in (float("nan"), float("inf"), -float("inf")):
        X = torch.where(k == 0, bad, 1.0).float()
        Y, S, s2, Z = (torch.empty_like(X) for _ in range(4))
        one = torch.ones_like(X)
        hch.hch_dropout_fwd(hch.HCH_F32, X, None, hch.HCH_F32, Y, n, c, p, 11)
        hch.hch_dropout_layernorm_fwd(hch.HCH_F32, X, one, S, None, None, hch.HCH_F32, Z, None, n, c, 1e-5, p, 11)
        assert torch.equal(Y, k.float()) and torch.equal(S, 1 + k.float()) and Z.isfinite().all()


def test_rows_beyond_32_bits():
    """More than 2^32 blocks and elements: a mask of one channel a row, the last rows."""
    n = 2 ** 32 + 4099
    X = torch.ones((n, 1), dtype=torch.bfloat16, device="cuda")
    hch.hch_dropout_fwd(hch.HCH_BF16, X, None, hch.HCH_BF16, X, n, 1, 0.5, 123)
    for first in (0, 2 ** 31 - 8, 2 ** 32 - 8, n - 300):
        want = R.dropout_factors(300, 1, 0.5, 123, first_row=first)
        assert (X[first: first + 300].double().cpu().numpy() == want).all()
    del X
    torch.cuda.empty_cache()


CHANNELS = [1, 2, 3, 4, 8, 16, 17, 50, 64, 100, 128, 200, 250, 256, 260, 512, 515, 1000, 1024, 1030, 2048, 2049, 2050, 4096, 4097, 8190, 8191, 8192]


@pytest.mark.parametrize("x,y,dx", [("f32", "f32", "f32"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32")])
@pytest.mark.parametrize("c", CHANNELS)
def test_dropout_with_sum_and_norm(x, y, dx, c):
    rng = np.random.default_rng(c)
    eps = 1e-5
    for n, p, affine, offset in ((1, 0.1, False, 0), (1030 if c <= 256 else 71, 0.2, True, 0), (33, 0.5, True, 1)):
        seed, step = int(rng.integers(0, 2 ** 63)), int(rng.integers(0, 2 ** 62))
        at = _step(step)
        X, xs = _on(rng, (n, c), x, offset)
        Rr, rs_ = _on(rng, (n, c), x, offset)
        g, gs = _on(rng, (c,), "f32") if affine else (None, None)
        b, bs = _on(rng, (c,), "f32") if affine else (None, None)
        S, Y = torch.empty_like(X), torch.empty((n, c), dtype=TYPES[y][1], device="cuda")
        stats = torch.empty((n, 2), device="cuda")
        hch.hch_dropout_layernorm_fwd(TYPES[x][0], X, Rr, S, g, b, TYPES[y][0], Y, stats, n, c, eps, p, seed, at)
        k = R.dropout_factors(n, c, p, seed, step)
        s, want, wstats = K.layernorm_fwd(k * xs, rs_, gs, bs, eps)
        es = 2 * U * np.abs(k * xs) + U * np.abs(s)                         # of s before it is rounded to its type
        _near(S, s, es + HALF[x] * (np.abs(s) + es), "s")
        size = (np.abs(s) + es).max(1, keepdims=True)
        dev = wstats[:, 1:]
        ga, ba = (np.abs(gs) if affine else 1.0), (np.abs(bs) if affine else 0.0)
        h = np.abs((s - wstats[:, :1]) * dev)
        # mean((s + d)) - mean(s) = mean(d), |d| <= es: where k x and r cancel, es is more than any multiple of s
        dmean = (c + 8) * U * size + es.mean(1, keepdims=True)
        ds_ = dmean + es                                                    # of s - mean
        rel = (c + 16) * 2 * U + (ds_ ** 2).mean(1, keepdims=True) * dev ** 2 + 2 * dev * (ds_ * h).mean(1, keepdims=True)
        # (sums of squares that are all rounding: their size is eps there)
        bound = (ds_ * dev * (1 + rel) + rel * h) * ga + 8 * U * (h * ga + ba)
        _near(Y, want, bound + HALF[y] * (np.abs(want) + bound) + 1e-30, "y")
        _near(stats[:, :1], wstats[:, :1], dmean + 1e-30, "mean")
        _near(stats[:, 1:], dev, rel * dev + 1e-30, "1 / deviation")

        DY, dys = _on(rng, (n, c), y, offset)
        DS, dss = _on(rng, (n, c), x, offset) if affine else (None, 0.0)
        srcs, st = S.double().cpu().numpy(), stats.double().cpu().numpy()
        dR, dX = torch.empty_like(X), torch.full((n, c), float("nan"), dtype=TYPES[dx][1], device="cuda")
        dg, db = torch.full((c,), float("nan"), device="cuda"), torch.full((c,), float("nan"), device="cuda")
        ws = torch.full((hch.hch_layernorm_workspace_bytes(n, c),), 255, dtype=torch.uint8, device="cuda")
        call = lambda dR, dX, dg, db, DS=DS: hch.hch_dropout_layernorm_bwd(TYPES[x][0], S, stats, g, TYPES[y][0], DY, DS, dR, TYPES[dx][0], dX, dg, db,
                                                                           n, c, p, seed, at, ws if dg is not None else None)
        call(dR, dX, dg, db)
        wdr, wdg, wdb = K.layernorm_bwd(srcs, st, gs, dys, dss if affine else None)
        h = (np.abs(srcs) + np.abs(st[:, :1])) * st[:, 1:]                  # sizes of what the differences are taken of
        w = np.abs(dys) * ga
        terms = st[:, 1:] * (w + w.mean(1, keepdims=True) + h * (w * h).mean(1, keepdims=True))
        err = (c + 16) * 2 * U * terms + 4 * U * np.abs(wdr) + U * np.abs(dss)
        _near(dR, wdr, err + HALF[x] * (np.abs(wdr) + err) + 1e-30, "dr")
        ex = k * (err + 2 * U * np.abs(wdr) * (1 + U))
        _near(dX, k * wdr, ex + HALF[dx] * (np.abs(k * wdr) + ex) + 1e-30, "dx")
        _near(dg, wdg, (n + 16) * U * (np.abs(dys) * h).sum(0) + 1e-30, "dgamma")
        _near(db, wdb, (n + 16) * U * np.abs(dys).sum(0) + 1e-30, "dbeta")
        assert ((dX == 0).cpu().numpy() >= (k == 0)).all()
        # the same bits again; without the weights' gradient; with dS in dR's place; S in X's and in R's
        dR2, dX2, dg2, db2 = (torch.empty_like(t) for t in (dR, dX, dg, db))
        call(dR2, dX2, dg2, db2)
        assert torch.equal(dR, dR2) and torch.equal(dX, dX2) and torch.equal(dg, dg2) and torch.equal(db, db2)
        if DS is not None:
            over = DS.clone() if offset == 0 else DS
            call(over, dX2, None, None, DS=over)
            assert torch.equal(dR, over) and torch.equal(dX, dX2)
        for over in (X, Rr):
            a, r = X.clone(), Rr.clone()
            s2 = a if over is X else r
            y2 = torch.empty_like(Y)
            hch.hch_dropout_layernorm_fwd(TYPES[x][0], a, r, s2, g, b, TYPES[y][0], y2, None, n, c, eps, p, seed, at)
            if offset == 0:                                                 # another alignment may add up in another order
                assert torch.equal(s2, S) and torch.equal(y2, Y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [50, 64, 63, 1030, 4097])
def test_results_in_the_place_of_arguments(dtype, c):
    """The same bits as in tensors of their own: each lane has read what it overwrites."""
    rng = np.random.default_rng(c)
    code, n, p, seed = TYPES[dtype][0], 3001 if c < 100 else 301, 0.3, 2 ** 64 - 9
    (X, _), (Rr, _), (DY, _), (DS, _) = (_on(rng, (n, c), dtype) for _ in range(4))
    at, stats = _step(7), torch.empty((n, 2), device="cuda")
    new = lambda: torch.full((n, c), float("nan"), dtype=TYPES[dtype][1], device="cuda")

    want = new()
    hch.hch_dropout_bwd(code, DY, code, want, n, c, p, seed, at)
    Z = DY.clone()
    hch.hch_dropout_bwd(code, Z, code, Z, n, c, p, seed, at)                # dx = dy
    assert torch.equal(Z, want)

    S, Y = new(), new()
    hch.hch_dropout_layernorm_fwd(code, X, Rr, S, None, None, code, Y, stats, n, c, 1e-5, p, seed, at)
    for k in range(2):                                                      # y = x, y = r; and s in the other's place
        for s_there in (False, True):
            a, r = X.clone(), Rr.clone()
            y, s = (a, r) if k == 0 else (r, a)
            s = s if s_there else new()
            hch.hch_dropout_layernorm_fwd(code, a, r, s, None, None, code, y, None, n, c, 1e-5, p, seed, at)
            assert torch.equal(y, Y) and torch.equal(s, S)

    dR, dX, dg, db = new(), new(), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = torch.full((hch.hch_layernorm_workspace_bytes(n, c),), 255, dtype=torch.uint8, device="cuda")
    hch.hch_dropout_layernorm_bwd(code, S, stats, None, code, DY, DS, dR, code, dX, dg, db, n, c, p, seed, at, ws)
    for k in range(3):                                                      # dr = s, dy, ds
        s, dy, ds = S.clone(), DY.clone(), DS.clone()
        r2, x2, dg2, db2 = (s, dy, ds)[k], new(), torch.empty_like(dg), torch.empty_like(db)
        hch.hch_dropout_layernorm_bwd(code, s, stats, None, code, dy, ds, r2, code, x2, dg2, db2, n, c, p, seed, at, ws)
        assert torch.equal(r2, dR) and torch.equal(x2, dX) and torch.equal(dg2, dg) and torch.equal(db2, db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,c", [(100003, 50), (100003, 64), (200001, 3), (20011, 250), (3001, 1030), (2003, 4097)])
def test_sums_over_many_rows_are_exact_where_they_are_whole(dtype, n, c):
    """Rows of +-1 that are normalised already (mean 0, deviation 1) and dy of 1 .. 7 with their sign, or all positive: every term of a
    sum is a positive whole number and sums stay below 2^24, so that they are exact in any order, and a row lost, taken twice or taken for
    another's shows."""
    rng = np.random.default_rng(n + c)
    sign = torch.from_numpy(rng.choice([-1.0, 1.0], (n, c)).astype(np.float32))
    size = torch.from_numpy(rng.integers(1, 8, (n, c)).astype(np.float32))
    S = sign.to(TYPES[dtype][1]).cuda()
    stats = torch.tensor([0.0, 1.0], device="cuda").repeat(n, 1)
    dR, dX = torch.empty_like(S), torch.empty_like(S)
    dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = torch.full((hch.hch_layernorm_workspace_bytes(n, c),), 255, dtype=torch.uint8, device="cuda")
    want = size.double().sum(0)
    for signed in (True, False):
        dY = (size * sign if signed else size).to(TYPES[dtype][1]).cuda()
        hch.hch_dropout_layernorm_bwd(TYPES[dtype][0], S, stats, None, TYPES[dtype][0], dY, None, dR, TYPES[dtype][0], dX, dg, db, n, c, 0.1, 3, None, ws)
        assert torch.equal((dg if signed else db).double().cpu(), want)
        assert torch.equal((db if signed else dg).double().cpu(), (size * sign).double().sum(0))


def test_one_mask_in_all_calls():
    """Alone and with the norm, in every type and at every alignment."""
    for c in (24, 50, 63, 1026):
        n, p, seed = 130, 0.4, 99
        at = _step(12)
        masks = []
        for t in ("f32", "bf16"):
            for offset in (0, 1, 2, 4):
                X = torch.ones(n * c + offset, dtype=TYPES[t][1], device="cuda")[offset:].view(n, c)
                zero, S, Y, dX = torch.zeros_like(X), torch.empty_like(X), torch.empty_like(X), torch.empty_like(X)
                hch.hch_dropout_fwd(TYPES[t][0], X, None, TYPES[t][0], Y, n, c, p, seed, at)
                masks.append(Y != 0)
                stats = torch.empty((n, 2), device="cuda")
                hch.hch_dropout_layernorm_fwd(TYPES[t][0], X, zero, S, None, None, TYPES[t][0], Y, stats, n, c, 1e-5, p, seed, at)
                masks.append(S != 0)
                stats[:, 0], stats[:, 1] = 0.0, 0.0                         # dr = ds
                hch.hch_dropout_layernorm_bwd(TYPES[t][0], S, stats, None, TYPES[t][0], X, X, Y, TYPES[t][0], dX, None, None, n, c, p, seed, at, None)
                masks.append(dX != 0)
        want = torch.from_numpy(R.dropout_factors(n, c, p, seed, 12) != 0).cuda()
        assert all(torch.equal(m, want) for m in masks)


def test_nothing_to_do():
    e = torch.empty((0, 8), device="cuda")
    hch.hch_dropout_fwd(hch.HCH_F32, e, None, hch.HCH_F32, e.clone(), 0, 8, 0.1, 0)
    hch.hch_dropout_bwd(hch.HCH_F32, e, hch.HCH_F32, e.clone(), 0, 8, 0.1, 0)
    hch.hch_dropout_layernorm_fwd(hch.HCH_F32, e, e, e, None, None, hch.HCH_F32, e, None, 0, 8, 1e-5, 0.1, 0)
    dg, db = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    hch.hch_dropout_layernorm_bwd(hch.HCH_F32, e, e, None, hch.HCH_F32, e, None, e, hch.HCH_F32, e.clone(), dg, db, 0, 8, 0.1, 0, None, ws)
    torch.cuda.synchronize()
    assert not dg.any() and not db.any()


@pytest.mark.parametrize("c", [50, 64])
def test_replayed_graphs_have_new_masks(c):
    n, p, seed = 500, 0.3, 5
    X, Rr = torch.randn((n, c), device="cuda"), torch.randn((n, c), device="cuda")
    dY = torch.randn((n, c), device="cuda")
    S, Y, D, dR, dX = (torch.empty_like(X) for _ in range(5))
    stats, dg, db = torch.empty((n, 2), device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = torch.empty(hch.hch_layernorm_workspace_bytes(n, c), dtype=torch.uint8, device="cuda")
    step = _step(0)

    def work():
        hch.hch_dropout_fwd(hch.HCH_F32, X, Rr, hch.HCH_F32, D, n, c, p, seed, step)
        hch.hch_dropout_layernorm_fwd(hch.HCH_F32, X, Rr, S, None, None, hch.HCH_F32, Y, stats, n, c, 1e-5, p, seed, step)
        hch.hch_dropout_layernorm_bwd(hch.HCH_F32, S, stats, None, hch.HCH_F32, dY, dY, dR, hch.HCH_F32, dX, dg, db, n, c, p, seed, step, ws)
        step.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    outs = (D, S, Y, stats, dR, dX, dg, db)
    seen = []
    for i in range(4):
        step.fill_(40 + i)
        X.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert int(step) == 41 + i
        step.fill_(40 + i)
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
        seen.append(dX != 0)
    assert all(not torch.equal(seen[0], s) for s in seen[1:])
