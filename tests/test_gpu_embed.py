"""hch_embed_fwd / _bwd against the 64-bit oracle.

Bounds: a row of the table times the scale is off by two roundings of fp32, and half a step where it is stored in bf16 (2^-8); a sum of m
rows in fp32, in whatever order, by m 2^-24 of the sum of their sizes."""
import numpy as np
import pytest

from oracle import rows as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
hch = pytest.importorskip("paper_1803_11385_amd")

TYPES = {"f32": (hch.HCH_F32, torch.float32), "bf16": (hch.HCH_BF16, torch.bfloat16)}
U = 2.0 ** -24
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}


def _rows(rng, n, c, ld, offset, dtype):
    x = torch.from_numpy(rng.normal(size=(n, c)).astype(np.float32)).to(TYPES[dtype][1])
    whole = torch.full((n * ld + offset,), -7.0, dtype=x.dtype, device="cuda")
    t = whole[offset:].view(n, ld)[:, :c]
    t.copy_(x)
    return t, x.double().numpy(), whole


def _near(got, want, bound, what):
    torch.cuda.synchronize()
    off = np.abs(got.double().cpu().numpy() - want) - bound
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} of {off.size} beyond the bound, worst {off.max()}"


def _ws(n, c, vocab):
    return torch.full((hch.hch_embed_workspace_bytes(n, c, vocab),), 255, dtype=torch.uint8, device="cuda")


def _ids(rng, n, vocab, kind):
    if kind == "uniform":
        ids = rng.integers(0, vocab, n)
    elif kind == "skewed":
        ids = np.minimum((rng.random(n) ** 4 * vocab).astype(np.int64), vocab - 1)
    elif kind == "one":
        ids = np.full(n, vocab - 1)
    elif kind == "blocks":                                 # runs that begin and end on the borders of 64 rows
        ids = np.repeat(np.arange(n), 64)[:n] // 33 % vocab
    elif kind == "none":
        ids = rng.choice([-1, vocab, 2 ** 31 - 1, -2 ** 31], n)
    else:                                                  # a tenth without a label
        ids = np.where(rng.random(n) < 0.1, rng.choice([-1, vocab, 2 ** 31 - 1, -2 ** 31], n), rng.integers(0, vocab, n))
    return ids.astype(np.int32)


def _gradient(rng, ids, vocab, c, y, scale=1.5, ld_more=0, offset=0, table_offset=0):
    n = ids.size
    I = torch.from_numpy(ids).cuda()
    dY, dys, _ = _rows(rng, n, c, c + ld_more, offset, y)
    dead = (ids < 0) | (ids >= vocab)
    if dead.any():
        dY[torch.from_numpy(dead).cuda()] = float("nan")   # is not read
        dys[dead] = 0.0
    dT = torch.full((vocab * c + table_offset,), float("nan"), device="cuda")[table_offset:].view(vocab, c)
    ws = _ws(n, c, vocab)
    hch.hch_embed_bwd(I, TYPES[y][0], dY, dT, n, c, vocab, scale, ws)
    want, size, count = R.embed_bwd(ids, dys, vocab, scale)
    _near(dT, want, (count[:, None] + 2) * U * size, f"dtable of {n} rows, {vocab} labels, {c} channels")
    again = torch.empty_like(dT)
    if table_offset == 0:
        ws.fill_(17)
        hch.hch_embed_bwd(I, TYPES[y][0], dY, again, n, c, vocab, scale, ws)
        assert torch.equal(again, dT)


@pytest.mark.parametrize("t,y", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("c", [1, 2, 3, 4, 5, 8, 12, 50, 64, 100, 250, 256, 260, 1030, 4096])
def test_rows_and_gradient_of_every_width(t, y, c):
    rng = np.random.default_rng(c)
    for n, vocab, scale in ((1, 1, 1.0), (70, 9, -0.3), (3000 if c <= 260 else 150, 50, c ** 0.5)):
        table, ts, _ = _rows(rng, vocab, c, c, 0, t)
        ids = _ids(rng, n, vocab, "gaps")
        guard = torch.full((n * c + 64,), 7.0, dtype=TYPES[y][1], device="cuda")
        Y = guard[: n * c].view(n, c)
        hch.hch_embed_fwd(TYPES[t][0], table, torch.from_numpy(ids).cuda(), TYPES[y][0], Y, n, c, vocab, scale)
        want = R.embed(ts, ids, scale)
        _near(Y, want, (2 * U + HALF[y] * (1 + 2 * U)) * np.abs(want), "y")
        assert (guard[n * c:] == 7).all()
        if t == y or t == "f32":
            _gradient(rng, ids, vocab, c, y, scale)


@pytest.mark.parametrize("kind", ["uniform", "skewed", "one", "blocks", "none", "gaps"])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 128, 2047, 2048, 2049, 4096, 4097, 8193, 20000])
def test_gradient_of_every_length(kind, n):
    rng = np.random.default_rng(n)
    for vocab in (1, 2, 50, 64, 65, 256, 513, 5000, 70000):
        _gradient(rng, _ids(rng, n, vocab, kind), vocab, 12, "f32")
    _gradient(rng, _ids(rng, n, 66, kind), 66, 3, "f32")
    _gradient(rng, _ids(rng, n, 300, kind), 300, 40, "bf16")


@pytest.mark.parametrize("vocab", [3, 63, 64, 65, 127, 128, 129, 511, 512, 513, 65535, 65537, 262144, 262145, 1000000, 20000000])
def test_tables_of_every_size(vocab):
    rng = np.random.default_rng(vocab)
    ids = _ids(rng, 30000, vocab, "uniform")
    ids[:3] = (0, vocab - 1, vocab // 2)
    _gradient(rng, ids, vocab, 4 if vocab > 10 ** 6 else 16, "f32")


@pytest.mark.parametrize("kind,vocab", [("one", 1), ("one", 700), ("skewed", 50), ("skewed", 65), ("gaps", 70), ("skewed", 40000), ("gaps", 2), ("blocks", 10 ** 5)])
@pytest.mark.parametrize("y,c", [("f32", 20), ("bf16", 64), ("f32", 7), ("bf16", 16), ("bf16", 6), ("f32", 1), ("f32", 200)])
def test_long_runs(kind, vocab, y, c):
    rng = np.random.default_rng(3)
    for n in (64 * 33, 64 * 33 + 1, 64 * 64 - 1, 200001):
        _gradient(rng, _ids(rng, n, vocab, kind), vocab, c, y)


@pytest.mark.parametrize("kind,vocab", [("gaps", 3000), ("one", 40), ("skewed", 300000)])
def test_more_tiles_than_a_workgroup_counts(kind, vocab):
    rng = np.random.default_rng(5)
    _gradient(rng, _ids(rng, 8192 * 160 + 4321, vocab, kind), vocab, 3, "f32")


def _exact_gradient(rng, ids, vocab, c, y, scale=0.5):
    """Rows of 1 .. 7, positive, and a scale of a power of two: sums are whole numbers below 2^24 times the scale, exact in any order; a row lost, taken
    twice or under another's label shows, however long its run."""
    n = ids.size
    made = torch.Generator(device="cuda").manual_seed(int(rng.integers(2 ** 31)))
    rows = torch.randint(1, 8, (n, c), generator=made, device="cuda").float()
    assert 7 * n < 2 ** 24
    I = torch.from_numpy(ids).cuda()
    sums = torch.zeros((n + 1, c), dtype=torch.float64, device="cuda")
    by_label, order = torch.sort(I.long())
    torch.cumsum(rows[order].double(), 0, out=sums[1:])    # whole numbers: exact
    ends = torch.searchsorted(by_label, torch.arange(-1, vocab, device="cuda"), right=True)
    want = sums[ends[1:]] - sums[ends[:-1]]
    dT = torch.full((vocab, c), float("nan"), device="cuda")
    hch.hch_embed_bwd(I, TYPES[y][0], rows.to(TYPES[y][1]), dT, n, c, vocab, scale, _ws(n, c, vocab))
    wrong = (dT.double() != scale * want).any(1)
    assert not wrong.any(), f"{n} rows of {c}: {int(wrong.sum())} of {vocab} labels, the first {int(wrong.nonzero()[0])}"


@pytest.mark.parametrize("kind,vocab", [("one", 1), ("one", 700), ("skewed", 2), ("skewed", 65), ("gaps", 2), ("skewed", 40000), ("blocks", 10 ** 5)])
@pytest.mark.parametrize("y,c", [("f32", 20), ("bf16", 64), ("f32", 7), ("bf16", 16), ("f32", 1), ("f32", 200), ("f32", 257), ("bf16", 256)])
def test_long_runs_are_exact_where_sums_are_whole(kind, vocab, y, c):
    rng = np.random.default_rng(c)
    for n in (64 * 33 + 1, 200001):
        _exact_gradient(rng, _ids(rng, n, vocab, kind), vocab, c, y)


@pytest.mark.parametrize("kind,vocab", [("gaps", 3000), ("one", 40), ("skewed", 2), ("skewed", 300000)])
@pytest.mark.parametrize("y,c", [("f32", 3), ("bf16", 64)])
def test_many_tiles_are_exact_where_sums_are_whole(kind, vocab, y, c):
    """On both sides of the lines at which a thread of the sort has more rows and the tiles' counts are added up by a launch of their own."""
    rng = np.random.default_rng(c)
    for n in (163840, 163841, 327681, 655360, 655361, 8192 * 160 + 4321):
        _exact_gradient(rng, _ids(rng, n, vocab, kind), vocab, c, y)


@pytest.mark.parametrize("y,c", [("f32", 1030), ("bf16", 1030), ("f32", 1031), ("bf16", 2048)])
@pytest.mark.parametrize("kind,vocab", [("one", 3), ("skewed", 5)])
def test_long_runs_of_wide_rows_are_exact_where_sums_are_whole(kind, vocab, y, c):
    rng = np.random.default_rng(c)
    _exact_gradient(rng, _ids(rng, 40009, vocab, kind), vocab, c, y)


@pytest.mark.parametrize("y,n,c,rows,chains", [("bf16", 609323, 1030, 64, 1), ("f32", 200001, 1031, 64, 1), ("f32", 152343, 256, 64, 4), ("bf16", 2 ** 22, 64, 512, 16)])
def test_long_runs_of_like_rows(y, n, c, rows, chains):
    """All rows alike, with one label: what each addition rounds away has the same sign, so that errors add up.  A value passes 16 additions in a group's
    rows, 6 at most from group to group and 4 from wavefront to wavefront, 64 in a block of the join's chain, as many as that chain has blocks, and
    those that join the chains; then the scale."""
    vocab = 2
    row = torch.from_numpy((0.5 + np.random.default_rng(c).random(c)).astype(np.float32)).to(TYPES[y][1]).cuda()
    dY = row.expand(n, c).contiguous()
    ids = torch.ones(n, dtype=torch.int32, device="cuda")
    dT = torch.full((vocab, c), float("nan"), device="cuda")
    hch.hch_embed_bwd(ids, TYPES[y][0], dY, dT, n, c, vocab, 0.3, _ws(n, c, vocab))
    want = n * float(np.float32(0.3)) * row.double().cpu().numpy()
    parts = -(-n // rows)
    depth = 16 + 6 + 4 + 64 + -(-parts // (64 * chains)) + chains.bit_length() + 1
    _near(dT, np.stack([0 * want, want]), depth * U * np.stack([want, want]), "dtable")
    del dY
    torch.cuda.empty_cache()


@pytest.mark.parametrize("c,tile", [(4, 1024), (40, 256), (64, 256), (200, 64)])
def test_runs_at_the_borders_of_groups_wavefronts_and_tiles(c, tile):
    """Runs that begin and end before, on and behind the borders of 16 rows, of a wavefront's rows and of a workgroup's, in every
    combination of neighbours."""
    rng = np.random.default_rng(4)
    for vocab in (4, 90):
        for before in (0, 1, 15, 16, 17, tile // 4 - 1, tile // 4, tile // 4 + 1, tile - 1, tile, tile + 1):
            for length in (1, 2, 15, 16, 17, tile // 4, tile - 1, tile, tile + 1, 2 * tile - 1, 2 * tile, 3 * tile + 7):
                ids = np.concatenate([np.zeros(before), np.ones(length), np.full(77, 2)]).astype(np.int32)
                _gradient(rng, rng.permutation(ids), vocab, c, "f32")


@pytest.mark.parametrize("c", [4, 40, 200])
def test_nan_and_infinity_stay_with_their_label(c):
    """Labels of one row, of a few and of more than a tile, one of them bad: the others' sums are those without it, bit for bit."""
    rng = np.random.default_rng(8)
    n, vocab = 9000, 120
    ids = np.concatenate([rng.integers(0, 60, 5000), np.full(2500, 60), np.arange(61, 120), rng.integers(0, 120, n - 7559)]).astype(np.int32)
    ids = rng.permutation(ids)
    dY, _, _ = _rows(rng, n, c, c, 0, "f32")
    I = torch.from_numpy(ids).cuda()
    clean, dT, ws = torch.empty((vocab, c), device="cuda"), torch.empty((vocab, c), device="cuda"), _ws(n, c, vocab)
    hch.hch_embed_bwd(I, hch.HCH_F32, dY, clean, n, c, vocab, 1.0, ws)
    for bad in (0, 60, 100):
        for value in (float("nan"), float("inf")):
            X = dY.clone()
            X[I == bad] = value
            hch.hch_embed_bwd(I, hch.HCH_F32, X, dT, n, c, vocab, 1.0, ws)
            others = torch.arange(vocab, device="cuda") != bad
            assert torch.equal(dT[others], clean[others]) and not dT[bad].isfinite().any()


@pytest.mark.parametrize("ld_more,offset", [(4, 0), (8, 8), (1, 0), (2, 2), (0, 1), (3, 3)])
def test_columns_of_wider_rows(ld_more, offset):
    rng = np.random.default_rng(6)
    n, vocab = 500, 30
    for y in ("f32", "bf16"):
        for c in (16, 50):
            ids = _ids(rng, n, vocab, "gaps")
            table, ts, _ = _rows(rng, vocab, c, c, offset, "f32")
            Y, _, whole = _rows(rng, n, c, c + ld_more, offset, y)
            hch.hch_embed_fwd(hch.HCH_F32, table, torch.from_numpy(ids).cuda(), TYPES[y][0], Y, n, c, vocab, 2.0)
            want = R.embed(ts, ids, 2.0)
            _near(Y, want, (2 * U + HALF[y] * (1 + 2 * U)) * np.abs(want), "y")
            whole[offset:].view(n, c + ld_more)[:, :c] = -7.0
            assert (whole == -7).all()
            _gradient(rng, ids, vocab, c, y, ld_more=ld_more, offset=offset)
            _gradient(rng, ids, vocab, c, y, table_offset=1)


def test_nothing_to_do():
    dT = torch.full((9, 5), float("nan"), device="cuda")
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    e = torch.empty((0, 5), device="cuda")
    hch.hch_embed_bwd(ids, hch.HCH_F32, e, dT, 0, 5, 9, 1.0, _ws(0, 5, 9))
    hch.hch_embed_fwd(hch.HCH_F32, dT, ids, hch.HCH_F32, e, 0, 5, 9, 1.0)
    torch.cuda.synchronize()
    assert not dT.any()


def test_more_than_2_to_32_elements():
    n, c, vocab = 2 ** 26 + 77, 64, 3
    table = torch.randn((vocab, c), device="cuda").bfloat16()
    ids = (torch.arange(n, device="cuda") % vocab).to(torch.int32)
    Y = torch.empty((n, c), dtype=torch.bfloat16, device="cuda")
    hch.hch_embed_fwd(hch.HCH_BF16, table, ids, hch.HCH_BF16, Y, n, c, vocab, 1.0)
    for first in (0, 2 ** 25 - 50, n - 100):
        assert torch.equal(Y[first: first + 100], table[ids[first: first + 100].long()])
    # rows of small whole numbers: exact sums in fp32 where they stay below 2^24
    Y.zero_()
    Y[::1000003] = 1.0
    Y[n - 1] = 3.0
    dT = torch.empty((vocab, c), device="cuda")
    hch.hch_embed_bwd(ids, hch.HCH_BF16, Y, dT, n, c, vocab, 1.0, _ws(n, c, vocab))
    want = torch.zeros(vocab, dtype=torch.float64)
    for i in range(0, n, 1000003):
        want[i % vocab] += 1
    want[(n - 1) % vocab] += 3 - (1 if (n - 1) % 1000003 == 0 else 0)
    assert (dT.double().cpu() == want[:, None]).all()
    del Y, ids
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [3000, 20000])
def test_labels_of_28_bits_and_a_table_of_2_to_32_elements(n):
    """Four passes of the sort; rows of the table behind 2^32 elements."""
    vocab, c = 2 ** 27 + 12345, 32
    table = torch.zeros((vocab, c), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(n)
    ids = rng.integers(0, vocab, n // 2)
    ids = rng.permutation(np.concatenate([ids, ids[::-1], [vocab - 1, 0]])).astype(np.int32)
    I = torch.from_numpy(ids).cuda()
    rows = torch.randn((ids.size, c), device="cuda").bfloat16()
    table[I.long()] = rows                                 # of two rows with one label, one of them
    Y = torch.empty_like(rows)
    hch.hch_embed_fwd(hch.HCH_BF16, table, I, hch.HCH_BF16, Y, ids.size, c, vocab, 1.0)
    assert torch.equal(Y, table[I.long()])
    del table
    torch.cuda.empty_cache()
    dT = torch.full((vocab, 1), float("nan"), device="cuda")
    dY, dys, _ = _rows(rng, ids.size, 1, 1, 0, "f32")
    hch.hch_embed_bwd(I, hch.HCH_F32, dY, dT, ids.size, 1, vocab, 1.0, _ws(ids.size, 1, vocab))
    labels, where = np.unique(ids, return_inverse=True)
    want, size, count = R.embed_bwd(where, dys, labels.size, 1.0)
    at = torch.from_numpy(labels).cuda().long()
    _near(dT[at], want, (count[:, None] + 2) * U * size, "dtable")
    dT[at] = 0.0
    assert not dT.any()                                    # NaN counts as something
    del dT
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,vocab", [(300, 20), (20000, 5000)])
def test_replayed_graph_and_another_stream(n, vocab):
    c = 24
    rng = np.random.default_rng(1)
    ids = torch.from_numpy(_ids(rng, n, vocab, "gaps")).cuda()
    table = torch.randn((vocab, c), device="cuda")
    Y, dT, ws = torch.empty((n, c), device="cuda"), torch.empty_like(table), _ws(n, c, vocab)

    def work():
        hch.hch_embed_fwd(hch.HCH_F32, table, ids, hch.HCH_F32, Y, n, c, vocab, 3.0)
        hch.hch_embed_bwd(ids, hch.HCH_F32, Y, dT, n, c, vocab, 0.5, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(4):
        ids.copy_(torch.from_numpy(_ids(rng, n, vocab, ("gaps", "one", "skewed", "none")[k])))
        table.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = Y.clone(), dT.clone()
        work()
        torch.cuda.synchronize()
        assert torch.equal(got[0], Y) and torch.equal(got[1], dT)
