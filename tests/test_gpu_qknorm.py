"""hch_qknorm_rope_* against the 64-bit oracle.

Bounds: a sum of d squares is off by (d + 4) 2^-24 of itself, its root by half of that; a turned pair by 2^-22 of its length; results in bf16 are
rounded once more, by half a step, 2^-8.  The gradient's terms carry these errors through its formula."""
import numpy as np
import pytest

from oracle import block as K
from oracle import rows as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
hch = pytest.importorskip("paper_1803_11385_amd")

TYPES = {"f32": (hch.HCH_F32, torch.float32), "bf16": (hch.HCH_BF16, torch.bfloat16)}
U = 2.0 ** -24
TURN = 2.0 ** -22
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}
EPS = 1e-5


def _rows(rng, n, width, ld, offset, dtype, gain=None):
    """n rows of `width` in rows of ld, `offset` elements behind a 256-byte border; what lies between them is -7."""
    x = rng.normal(size=(n, width)).astype(np.float32)
    if gain is not None:
        x = x * gain
    x = torch.from_numpy(x).to(TYPES[dtype][1])
    whole = torch.full((n * ld + offset,), -7.0, dtype=x.dtype, device="cuda")
    t = whole[offset:].view(n, ld)[:, :width]
    t.copy_(x)
    return t, x.double().numpy(), whole


def _near(got, want, bound, what):
    torch.cuda.synchronize()
    off = np.abs(got.double().cpu().numpy() - want) - bound
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} of {off.size} beyond the bound, worst {off.max()}"


def _lengths(a, d):
    """of the pair that each channel belongs to"""
    z = a.reshape(a.shape[0], -1, d // 2, 2)
    return np.repeat(np.sqrt((z ** 2).sum(3, keepdims=True)), 2, 3).reshape(a.shape)


def _check(rng, n, heads, hq, hk, d, sections, x, y, dx, ld_more=0, offset=0, gammas=True, u=64, base=10000.0, scale=1.0):
    w = heads * d
    gain = np.repeat(np.exp(rng.normal(size=(1, heads))), d, 1).astype(np.float32)
    X, xs, _ = _rows(rng, n, w, w + ld_more, offset, x, gain)
    gq = rng.normal(size=d).astype(np.float32) if gammas else None
    gk = rng.normal(size=d).astype(np.float32) if gammas else None
    on = lambda a: None if a is None else torch.from_numpy(a).cuda()
    pos = rng.integers(0, u, (n, 3)).astype(np.int32)
    co = on(pos)
    Y, _, whole = _rows(rng, n, w, w + ld_more, offset, y)
    Y.fill_(float("nan"))
    hch.hch_qknorm_rope_fwd(TYPES[x][0], X, TYPES[y][0], Y, on(gq), on(gk), co, n, heads, hq, hk, d, sections, base, scale, EPS)
    scale = float(np.float32(scale))                        # the call takes it as fp32: at a million voxels 2^-25 of it is a hundredth of a turn
    want = R.qknorm_rope(xs, gq, gk, pos, heads, hq, hk, d, sections, base, scale, EPS)
    turned = (hq + hk) * d
    err = ((d / 2 + 12) * U + TURN) * _lengths(want, d)
    err[:, turned:] = 0.0
    _near(Y, want, err + HALF[y] * (np.abs(want) + err) * (1 if x != y else np.arange(w) < turned), "y")
    between = whole.clone()
    between[offset:].view(n, w + ld_more)[:, :w] = -7.0
    assert (between == -7).all()
    if x == y:                                              # in place: the same bits, values' heads as they were
        Z = X.clone() if not ld_more and not offset else None
        if Z is not None:
            hch.hch_qknorm_rope_fwd(TYPES[x][0], Z, TYPES[y][0], Z, on(gq), on(gk), co, n, heads, hq, hk, d, sections, base, scale, EPS)
            assert torch.equal(Z, Y)

    dY, dys, _ = _rows(rng, n, w, w + ld_more, offset, y)
    dX, _, whole = _rows(rng, n, w, w + ld_more, offset, dx)
    dX.fill_(float("nan"))
    dgq, dgk = torch.full((d,), float("nan"), device="cuda"), torch.full((d,), float("nan"), device="cuda")
    ws = torch.full((hch.hch_qknorm_rope_workspace_bytes(n, hq, hk, d),), 255, dtype=torch.uint8, device="cuda")

    def back(dY, dX, dgq, dgk, ws=ws):
        hch.hch_qknorm_rope_bwd(TYPES[x][0], X, TYPES[y][0], dY, TYPES[dx][0], dX, on(gq), on(gk), dgq, dgk, co, n, heads, hq, hk, d, sections, ws, base,
                                scale, EPS)
    back(dY, dX, dgq, dgk)
    wdx, wdq, wdk, size = R.qknorm_rope_bwd(xs, dys, gq, gk, pos, heads, hq, hk, d, sections, base, scale, EPS)
    dz = K.rope(dys, pos, heads, hq + hk, d, sections, base, scale, inverse=True).reshape(n, heads, d)
    ez = TURN * _lengths(dys, d).reshape(n, heads, d)
    z = xs.reshape(n, heads, d)
    r = 1.0 / np.sqrt((z ** 2).mean(2, keepdims=True) + EPS)
    v = np.abs(z) * r
    g = np.ones((heads, d))
    if gammas:
        g[:hq], g[hq: hq + hk] = np.abs(gq), np.abs(gk)
    wa, we = np.abs(dz) * g, ez * g
    mean = lambda a: a.mean(2, keepdims=True)
    err = r * (we + v * mean(we * v) + (2 * d + 32) * U * (wa + v * mean(wa * v)))
    err[:, hq + hk:] = 0.0
    err = err.reshape(n, w)
    _near(dX, wdx, err + HALF[dx] * (np.abs(wdx) + err) * (1 if y != dx else np.arange(w) < turned), "dx")
    for k, (got, want, first, count) in enumerate(((dgq, wdq, 0, hq), (dgk, wdk, hq, hk))):
        lost = (ez * v)[:, first: first + count].sum((0, 1))
        _near(got, want, (n * count + d + 32) * U * (size[k] + lost) + lost + 1e-30, ("dgamma_q", "dgamma_k")[k])
    between = whole.clone()
    between[offset:].view(n, w + ld_more)[:, :w] = -7.0
    assert (between == -7).all()
    # the same bits again, without the weights' gradient, and in place
    again, a, b = torch.empty_like(dX), torch.empty_like(dgq), torch.empty_like(dgk)
    if not ld_more and not offset:
        back(dY, again, a, b)
        assert torch.equal(again, dX) and torch.equal(a, dgq) and torch.equal(b, dgk)
        again.zero_()
        back(dY, again, None, None, None)
        assert torch.equal(again, dX)
        if y == dx:
            Z = dY.clone()
            back(Z, Z, None, None, None)
            assert torch.equal(Z, dX)


ALL = [("f32", "f32", "f32"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "bf16"), ("f32", "bf16", "f32"), ("bf16", "bf16", "f32")]


@pytest.mark.parametrize("x,y,dx", ALL)
@pytest.mark.parametrize("d", [2, 4, 6, 8, 14, 16, 24, 32, 34, 40, 48, 64, 66, 96, 128, 130, 250, 256])
def test_every_width(x, y, dx, d):
    rng = np.random.default_rng(d)
    third = d // 6
    for n, hq, hk, hv in ((1, 1, 1, 0), (7, 4, 2, 2), (300, 3, 1, 1)):
        _check(rng, n, hq + hk + hv, hq, hk, d, (d // 2 - 2 * third, third, third), x, y, dx)


@pytest.mark.parametrize("x,y,dx", ALL[:4])
@pytest.mark.parametrize("ld_more,offset", [(8, 0), (4, 4), (2, 0), (1, 0), (0, 1), (0, 2), (3, 3)])
def test_strides_and_alignments(x, y, dx, ld_more, offset):
    rng = np.random.default_rng(5)
    for d in (32, 40):
        _check(rng, 45, 5, 2, 2, d, (5, 5, 5), x, y, dx, ld_more, offset)


@pytest.mark.parametrize("heads,hq,hk", [(1, 1, 0), (1, 0, 1), (1, 0, 0), (3, 0, 2), (17, 16, 1), (48, 16, 16), (300, 200, 50)])
def test_head_counts(heads, hq, hk):
    rng = np.random.default_rng(heads)
    for x, y, dx in ALL[:3]:
        _check(rng, 33, heads, hq, hk, 16, (3, 3, 2), x, y, dx)
    _check(rng, 2500, heads if heads < 20 else 3, min(hq, 2), min(hk, 1), 8, (2, 1, 1), "f32", "f32", "f32")


def test_positions_far_away_partial_sections_and_no_gammas():
    rng = np.random.default_rng(9)
    for sections in ((0, 0, 0), (1, 0, 0), (0, 0, 16), (3, 2, 1), (8, 4, 4)):
        _check(rng, 50, 4, 2, 1, 32, sections, "f32", "f32", "f32", gammas=False, u=1000000, base=100.0, scale=-0.37)


def test_longer_than_one_wave_of_workgroups():
    _check(np.random.default_rng(2), 30011, 3, 1, 1, 64, (12, 10, 10), "bf16", "bf16", "bf16")
    _check(np.random.default_rng(2), 30011, 4, 2, 1, 20, (4, 3, 3), "f32", "bf16", "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,heads,hq,hk,d", [(1, 3, 1, 1, 64), (45, 5, 2, 2, 40), (3001, 6, 3, 1, 32), (2000, 3, 2, 1, 66), (5000, 4, 0, 2, 16)])
@pytest.mark.parametrize("ld_more,offset", [(0, 0), (16, 0), (4, 4), (2, 2), (3, 1)])
def test_results_in_the_place_of_arguments(dtype, n, heads, hq, hk, d, ld_more, offset):
    """The same bits as in tensors of their own, also in columns of wider rows, whose other columns stay."""
    rng = np.random.default_rng(n)
    w, ld, code = heads * d, heads * d + ld_more, TYPES[dtype][0]
    sections = (d // 2 - 2 * (d // 6), d // 6, d // 6)
    gq, gk = torch.randn(d, device="cuda"), torch.randn(d, device="cuda")
    co = torch.from_numpy(rng.integers(0, 64, (n, 3)).astype(np.int32)).cuda()
    ws = torch.full((hch.hch_qknorm_rope_workspace_bytes(n, hq, hk, d),), 255, dtype=torch.uint8, device="cuda")
    place = (co, n, heads, hq, hk, d, sections)

    def rows():
        t, _, whole = _rows(rng, n, w, ld, offset, dtype)
        return t, whole

    def twin(whole):
        whole = whole.clone()
        return whole[offset:].view(n, ld)[:, :w], whole

    def rest_stays(whole):
        between = whole.clone()
        between[offset:].view(n, ld)[:, :w] = -7.0
        assert (between == -7).all()

    (X, xw), (dY, yw), (Y, _) = rows(), rows(), rows()
    hch.hch_qknorm_rope_fwd(code, X, code, Y, gq, gk, *place)
    Z, zw = twin(xw)
    hch.hch_qknorm_rope_fwd(code, Z, code, Z, gq, gk, *place)
    assert torch.equal(Z, Y)
    rest_stays(zw)

    dX, _ = rows()
    dg = [torch.full((d,), float("nan"), device="cuda") for _ in range(2)]
    hch.hch_qknorm_rope_bwd(code, X, code, dY, code, dX, gq, gk, *dg, *place, ws)
    assert dX.isfinite().all()
    for over in ("dY", "X"):
        (x, x_), (dy, y_) = twin(xw), twin(yw)
        out, whole = (dy, y_) if over == "dY" else (x, x_)
        got = [torch.full((d,), float("nan"), device="cuda") for _ in range(2)]
        hch.hch_qknorm_rope_bwd(code, x, code, dy, code, out, gq, gk, *got, *place, ws)
        assert torch.equal(out, dX), over
        rest_stays(whole)
        # in dY's place values' heads are not walked through, so that rows may be in other workgroups: both orders have no more than 64 terms in a lane,
        # 64 groups of lanes and 40 sums of workgroups behind each other
        u = X.double().cpu().numpy().reshape(n, heads, d)
        u = np.abs(u) / np.sqrt((u ** 2).mean(2, keepdims=True) + EPS)
        terms = u * _lengths(dY.double().cpu().numpy(), d).reshape(n, heads, d)
        for a, b, first, count in zip(got, dg, (0, hq), (hq, hk)):
            assert torch.equal(a, b) if over == "X" else True
            _near(a, b.double().cpu().numpy(), 2 * 168 * U * terms[:, first: first + count].sum((0, 1)), "dgamma")


@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("n,heads,hq,hk,d", [(30011, 3, 1, 1, 64), (30011, 6, 4, 2, 16), (200003, 2, 1, 1, 32), (50021, 3, 2, 0, 128), (20021, 4, 2, 1, 256)])
def test_sums_over_many_rows_are_exact_where_they_are_whole(x, y, n, heads, hq, hk, d):
    """Heads of +-1 without positions, eps 0: u = x.  dy is 1 .. 7 with the sign of x, so that every term of gamma's gradient is a positive whole
    number and sums stay below 2^24: exact in any order, and a head or row lost, taken twice or taken for another's shows."""
    rng = np.random.default_rng(n + d)
    sign = torch.from_numpy(rng.choice([-1.0, 1.0], (n, heads, d)).astype(np.float32))
    size = torch.from_numpy(rng.integers(1, 8, (n, heads, d)).astype(np.float32))
    X = sign.to(TYPES[x][1]).cuda().view(n, -1)
    dY = (size * sign).to(TYPES[y][1]).cuda().view(n, -1)
    dX = torch.empty_like(X)
    dgq, dgk = (torch.full((d,), float("nan"), device="cuda") for _ in range(2))
    co = torch.zeros((n, 3), dtype=torch.int32, device="cuda")
    ws = torch.full((hch.hch_qknorm_rope_workspace_bytes(n, hq, hk, d),), 255, dtype=torch.uint8, device="cuda")
    hch.hch_qknorm_rope_bwd(TYPES[x][0], X, TYPES[y][0], dY, TYPES[x][0], dX, None, None, dgq, dgk, co, n, heads, hq, hk, d, (0, 0, 0), ws, eps=0.0)
    assert torch.equal(dgq.double().cpu(), size[:, :hq].double().sum((0, 1)))
    assert torch.equal(dgk.double().cpu(), size[:, hq: hq + hk].double().sum((0, 1)))


def test_heads_of_zeros_and_tiny_ones():
    n, d = 6, 64
    X = torch.zeros((n, 3 * d), device="cuda")
    X[1] = 1e-30
    X[2, 5] = 1e15
    Y, co = torch.empty_like(X), torch.zeros((n, 3), dtype=torch.int32, device="cuda")
    hch.hch_qknorm_rope_fwd(hch.HCH_F32, X, hch.HCH_F32, Y, None, None, co, n, 3, 1, 1, d, (11, 11, 10), eps=1e-6)
    assert not Y[0].any() and Y.isfinite().all()
    want = R.qknorm_rope(X.double().cpu().numpy(), None, None, co.cpu().numpy(), 3, 1, 1, d, (11, 11, 10), 1e4, 1.0, 1e-6)
    _near(Y, want, ((d / 2 + 12) * U + TURN) * np.abs(want) + 1e-37, "y")
    dX = torch.empty_like(X)
    hch.hch_qknorm_rope_bwd(hch.HCH_F32, X, hch.HCH_F32, torch.ones_like(X), hch.HCH_F32, dX, None, None, None, None, co, n, 3, 1, 1, d, (11, 11, 10),
                            None, eps=1e-6)
    assert torch.allclose(dX[0, : 2 * d], torch.tensor(1e3, device="cuda")) and dX.isfinite().all()


@pytest.mark.parametrize("d", [16, 64, 66])
def test_nan_stays_in_its_head(d):
    rng = np.random.default_rng(d)
    n, heads, hq, hk = 70, 5, 2, 2
    X, _, _ = _rows(rng, n, heads * d, heads * d, 0, "f32")
    dY, _, _ = _rows(rng, n, heads * d, heads * d, 0, "f32")
    co = torch.from_numpy(rng.integers(0, 9, (n, 3)).astype(np.int32)).cuda()
    ws = torch.empty(hch.hch_qknorm_rope_workspace_bytes(n, hq, hk, d), dtype=torch.uint8, device="cuda")

    def both(X):
        Y, dX, dgq, dgk = torch.empty_like(X), torch.empty_like(X), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        args = (co, n, heads, hq, hk, d, (d // 6, d // 6, 1))
        hch.hch_qknorm_rope_fwd(hch.HCH_F32, X, hch.HCH_F32, Y, None, None, *args)
        hch.hch_qknorm_rope_bwd(hch.HCH_F32, X, hch.HCH_F32, dY, hch.HCH_F32, dX, None, None, dgq, dgk, *args, ws)
        return Y.view(n, heads, d), dX.view(n, heads, d), dgq, dgk

    want = both(X)
    for head in (1, 2):
        Z = X.clone()
        Z.view(n, heads, d)[17, head, 3] = float("nan")
        got = both(Z)
        rest = torch.ones((n, heads), dtype=torch.bool, device="cuda")
        rest[17, head] = False
        for a, b in zip(got[:2], want[:2]):
            assert torch.equal(a[rest], b[rest]) and a[17, head].isnan().all()
        assert torch.equal(got[3 - (head == 2)], want[3 - (head == 2)]) and got[2 + (head == 2)].isnan().all()


def test_agrees_with_the_positions_alone():
    """Where all rows have the size sqrt(d) and eps is 0, what is left is hch_rope_fwd."""
    n, heads, d = 77, 3, 48
    X = torch.randn((n, heads, d), device="cuda", dtype=torch.float64)
    X = (X / X.pow(2).mean(2, keepdim=True).sqrt()).float().view(n, -1)
    co = torch.randint(0, 512, (n, 3), device="cuda", dtype=torch.int32)
    a, b = torch.empty_like(X), torch.empty_like(X)
    hch.hch_rope_fwd(hch.HCH_F32, X, hch.HCH_F32, a, co, n, heads, 2, d, (8, 8, 8))
    hch.hch_qknorm_rope_fwd(hch.HCH_F32, X, hch.HCH_F32, b, None, None, co, n, heads, 2, 0, d, (8, 8, 8), eps=0.0)
    assert (a - b).abs().max() <= (d / 2 + 12) * U * 8 and torch.equal(a[:, 2 * d:], b[:, 2 * d:])


def test_nothing_to_do():
    e = torch.empty((0, 64), device="cuda")
    dgq, dgk = torch.ones(16, device="cuda"), torch.ones(16, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    hch.hch_qknorm_rope_fwd(hch.HCH_F32, e, hch.HCH_F32, e.clone(), None, None, None, 0, 4, 2, 1, 16, (2, 2, 2))
    hch.hch_qknorm_rope_bwd(hch.HCH_F32, e, hch.HCH_F32, e.clone(), hch.HCH_F32, e.clone(), None, None, dgq, dgk, None, 0, 4, 2, 1, 16, (2, 2, 2), ws)
    torch.cuda.synchronize()
    assert not dgq.any() and not dgk.any()


def test_rows_beyond_32_bits():
    """2^32 elements and more: the last rows."""
    n, heads, d = 2 ** 22 + 5, 16, 64
    X = torch.empty((n, heads * d), dtype=torch.bfloat16, device="cuda")
    X.view(-1)[: 2 ** 26].normal_()
    X[-300:].normal_()
    co = torch.randint(0, 512, (n, 3), device="cuda", dtype=torch.int32)
    keep = X[-300:].clone()
    hch.hch_qknorm_rope_fwd(hch.HCH_BF16, X, hch.HCH_BF16, X, None, None, co, n, heads, 8, 4, d, (12, 10, 10))
    want = R.qknorm_rope(keep.double().cpu().numpy(), None, None, co[-300:].cpu().numpy(), heads, 8, 4, d, (12, 10, 10), 1e4, 1.0, EPS)
    _near(X[-300:], want, (HALF["bf16"] + TURN + 50 * U) * _lengths(want, d), "y")
    del X
    torch.cuda.empty_cache()


def test_replayed_graph_and_another_stream():
    n, heads, d = 400, 4, 32
    X, dY = torch.randn((n, heads * d), device="cuda"), torch.randn((n, heads * d), device="cuda")
    gq, gk = torch.randn(d, device="cuda"), torch.randn(d, device="cuda")
    co = torch.randint(0, 64, (n, 3), device="cuda", dtype=torch.int32)
    Y, dX, dgq, dgk = torch.empty_like(X), torch.empty_like(X), torch.empty_like(gq), torch.empty_like(gk)
    ws = torch.empty(hch.hch_qknorm_rope_workspace_bytes(n, 2, 1, d), dtype=torch.uint8, device="cuda")

    def work():
        hch.hch_qknorm_rope_fwd(hch.HCH_F32, X, hch.HCH_F32, Y, gq, gk, co, n, heads, 2, 1, d, (6, 5, 5))
        hch.hch_qknorm_rope_bwd(hch.HCH_F32, X, hch.HCH_F32, dY, hch.HCH_F32, dX, gq, gk, dgq, dgk, co, n, heads, 2, 1, d, (6, 5, 5), ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(4):
        X.normal_()
        gq.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, dX, dgq, dgk)]
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (Y, dX, dgq, dgk)))
