"""pipeline.AttentionBlock: norm, projections (convolutions with F = 1), rotary positions, attention and residual sum run
together on a level of a level set, forward and backward, against the same block in 64 bits on the CPU, whose
gradients are taken by automatic differentiation.  Bars as for the convolutions: 1e-4 of a value and its tensor's rms in
fp32, 2e-2 in bf16."""
import numpy as np
import pytest

import synth_shapes as S

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
hch = pytest.importorskip("paper_1803_11385_amd")


def _oracle(x, w, pos, off, mask, hq, hkv, d, sections, dy, ds):
    """The block in float64; returns results and gradients by name."""
    p = {k: v.double().cpu().requires_grad_(True) for k, v in dict(w, X=x).items()}

    def norm(t, i):
        m = t.mean(1, keepdim=True)
        return (t - m) / torch.sqrt(((t - m) ** 2).mean(1, keepdim=True) + 1e-5) * p[f"gamma{i}"] + p[f"beta{i}"]

    n = x.shape[0]
    qkv = (norm(p["X"], 0) @ p["Wqkv"]).reshape(n, hq + 2 * hkv, d // 2, 2)
    z = torch.view_as_complex(qkv.contiguous())
    ang = torch.cat([pos[:, a: a + 1].double() * 10000.0 ** (-torch.arange(s).double() / s) for a, s in enumerate(sections)], 1)
    ang = torch.cat([ang, torch.zeros(n, d // 2 - ang.shape[1])], 1)
    turn = torch.polar(torch.ones_like(ang), ang)[:, None, :]
    z = torch.cat([z[:, : hq + hkv] * turn, z[:, hq + hkv:]], 1)
    r = torch.view_as_real(z).reshape(n, hq + 2 * hkv, d)
    q, k, v = r[:, :hq], r[:, hq: hq + hkv].repeat_interleave(hq // hkv, 1), r[:, hq + hkv:].repeat_interleave(hq // hkv, 1)
    out = []
    for b in range(len(off) - 1):
        sl = slice(off[b], off[b + 1])
        s = torch.einsum("ihd,jhd->hij", q[sl], k[sl]) * d ** -0.5
        if mask is not None:
            s = s.masked_fill(~mask[sl][None, None, :], float("-inf"))
        out.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), v[sl]).reshape(-1, hq * d))
    res = p["X"] + torch.cat(out) @ p["Wo"]
    y = norm(res, 1)
    ((y * dy.double().cpu()).sum() + (res * ds.double().cpu()).sum()).backward()
    return dict(S=res.detach(), Y=y.detach(), **{"d" + k: v.grad for k, v in p.items()})


@pytest.mark.parametrize("dtype,bar", [(hch.HCH_F32, 1e-4), (hch.HCH_BF16, 2e-2)])
@pytest.mark.parametrize("c,hq,hkv,d,masked", [(32, 4, 4, 16, False), (48, 4, 2, 32, True)])
def test_block_against_automatic_differentiation(dtype, bar, c, hq, hkv, d, masked):
    from paper_1803_11385_amd import pipeline
    coords, offs, _ = S.config_batch(2, batch=3, u=32)
    lv = hch.hch_build_levels(coords, offs, 32, 3)
    blk = pipeline.AttentionBlock(lv, 1, c, hq, hkv, d, dtype=dtype)
    n = blk.n
    rng = np.random.default_rng(7)
    t = torch.bfloat16 if dtype == hch.HCH_BF16 else torch.float32
    on = lambda *shape, by=1.0, to=torch.float32: torch.from_numpy((by * rng.normal(size=shape)).astype(np.float32)).to(to).cuda()
    w = dict(Wqkv=on(c, blk.wide, by=c ** -0.5, to=t), Wo=on(hq * d, c, by=(hq * d) ** -0.5, to=t), gamma0=1 + on(c, by=0.1),
             beta0=on(c, by=0.1), gamma1=1 + on(c, by=0.1), beta1=on(c, by=0.1))
    blk.Wqkv.copy_(w["Wqkv"][None])
    blk.Wo.copy_(w["Wo"][None])
    for i in range(2):
        blk.gamma[i].copy_(w[f"gamma{i}"])
        blk.beta[i].copy_(w[f"beta{i}"])
    x, dy, ds = on(n, c), on(n, c), on(n, c)
    blk.X.copy_(x)
    blk.dY.copy_(dy)
    mask = None
    if masked:
        mask = torch.from_numpy(rng.random(n) < 0.7)
        blk.key_mask = mask.to(torch.uint8).cuda()
    blk.forward()
    blk.backward(ds)
    torch.cuda.synchronize()
    want = _oracle(x, w, blk.positions.cpu(), blk.offsets.tolist(), mask, hq, hkv, d, blk.sections, dy, ds)
    got = dict(S=blk.S, Y=blk.Y, dX=blk.dX, dWqkv=blk.dWqkv[0], dWo=blk.dWo[0], dgamma0=blk.dgamma[0], dgamma1=blk.dgamma[1],
               dbeta0=blk.dbeta[0], dbeta1=blk.dbeta[1])
    for name, g in got.items():
        e = want[name]
        off = (g.double().cpu() - e).abs() / (e.abs() + e.pow(2).mean().sqrt())
        assert off.max() <= bar, f"{name}: {off.max():.2e} of {bar}"


@pytest.mark.parametrize("dtype,bar", [(hch.HCH_F32, 1e-4), (hch.HCH_BF16, 2e-2)])
@pytest.mark.parametrize("c", [33, 47, 34, 36])
def test_every_channel_count(monkeypatch, dtype, bar, c):
    """Widths that are multiples of nothing, 2 and 4; every buffer of the block holds NaN before the passes, so that an element that
    none of them writes shows."""
    from paper_1803_11385_amd import pipeline
    init = pipeline.AttentionBlock.__init__

    def poisoned(self, *args, **kw):
        init(self, *args, **kw)
        for name in ("S", "Y", "P", "h", "O", "proj", "qkv", "lse", "dX", "dS", "dh", "dP", "dO32", "dO", "dqkv", "dWqkv", "dWo"):
            getattr(self, name).fill_(float("nan"))

    monkeypatch.setattr(pipeline.AttentionBlock, "__init__", poisoned)
    test_block_against_automatic_differentiation(dtype, bar, c, 4, 2, 16, True)
