"""The operators of an attention block over the voxels of a level, as cases that can be timed: layer norm
(with the residual sum in front of it) and its gradients, rotary positions from voxel coordinates,
attention inside each shape of a ragged batch, and its training step.

`run` computes them in plain form (elementary torch operations in 32 bits, rounded once at the end), or,
where `own` is set, through the library's calls.  Rows are voxels, all shapes of a batch one after
the other; the sizes are those of the levels of the encoders that this package runs (voxel counts of
unions of surface shells at 16^3 .. 512^3, channels 4 .. 256)."""
from __future__ import annotations

import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # the last level of a single 32^3 shape that is classified while somebody waits: a norm of latency
        dict(name="ln_fwd_32x1", kind="ln_fwd", n=752, c=64, x="f32", y="f32", residual=False),
        # residual sum and norm over the finest level of the 256^3 batch of 8, handing bf16 rows on
        dict(name="ln_fwd_256x8", kind="ln_fwd", n=609323, c=64, x="f32", y="bf16", residual=True),
        # gradients at a width that is a multiple of nothing (the 50 part labels of a segmentation head), 64^3
        dict(name="ln_bwd_64x16", kind="ln_bwd", n=63331, c=50, x="f32", y="f32", residual=False),
        # gradients of bf16 training at 128^3, the residual path's gradient added
        dict(name="ln_bwd_128x16", kind="ln_bwd", n=279722, c=128, x="bf16", y="bf16", residual=True),
        # positions of a projected, packed QKV row at the 32^3 level of the 256^3 batch, fp32 in, bf16 on
        dict(name="rope_fwd_32x8", kind="rope", inverse=False, n=9533, u=32, x="f32", y="bf16", heads=12, rot=8, d=64,
             sx=11, sy=11, sz=10),
        # the gradient's way back through them at the 128^3 level, shared key heads, bf16
        dict(name="rope_bwd_128x8", kind="rope", inverse=True, n=152331, u=128, x="bf16", y="bf16", heads=12, rot=10, d=32,
             sx=5, sy=5, sz=5),
        # one learned query pools the voxels of one shape into a token: nothing but latency
        dict(name="pool_f32_32x1", kind="attn_fwd", dtype="f32", batch=1, n=752, queries=1, hq=4, hkv=4, d=16, keep=1.0),
        # the same over the finest voxels of 8 shapes at once, query heads in groups of four: a pass over the keys
        dict(name="pool_bf16_256x8", kind="attn_fwd", dtype="bf16", batch=8, n=609323, queries=1, hq=8, hkv=2, d=32, keep=1.0),
        # masked pre-training at the 16^3 level of the 64^3 mini-batch: ragged shapes, a quarter of the keys left
        # out, one shape without any, an odd width, shared key heads, fp32
        dict(name="attn_f32_16x32", kind="attn_fwd", dtype="f32", batch=32, n=7917, queries=0, hq=6, hkv=2, d=40, keep=0.75),
        # the largest forward pass: every voxel of the 64^3 level of the 512^3 batch sees its whole shape
        dict(name="attn_bf16_64x4", kind="attn_fwd", dtype="bf16", batch=4, n=46514, queries=0, hq=4, hkv=4, d=128, keep=1.0),
        # training step of the fp32 block at the 16^3 level of the 256^3 batch
        dict(name="train_f32_16x8", kind="attn_train", dtype="f32", batch=8, n=2381, queries=0, hq=8, hkv=8, d=32, keep=1.0),
        # training step in bf16 at the 64^3 level of that batch
        dict(name="train_bf16_64x8", kind="attn_train", dtype="bf16", batch=8, n=38083, queries=0, hq=8, hkv=4, d=64, keep=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ln_fwd", "ln_bwd", "rope", "pool", "attn_fwd", "attn_fwd", "attn_train", "attn_train"])
    if kind in ("ln_fwd", "ln_bwd"):
        c = rng.choice([4, 16, 32, 50, 64, 96, 128, 200, 256, 512])
        x = rng.choice(["f32", "bf16"])
        return dict(kind=kind, n=_log_int(rng, 300, min(610000, 36000000 // c)), c=c, x=x,
                    y=rng.choice(["f32", "bf16"]) if x == "f32" else "bf16", residual=rng.random() < 0.5)
    if kind == "rope":
        d = rng.choice([16, 32, 48, 64, 96, 128])
        hkv = rng.choice([1, 2, 4])
        hq = hkv * rng.choice([1, 2, 4])
        s = d // 6
        x = rng.choice(["f32", "bf16"])
        return dict(kind="rope", inverse=rng.random() < 0.5, n=_log_int(rng, 300, min(300000, 58000000 // ((hq + 2 * hkv) * d))),
                    u=rng.choice([16, 32, 64, 128, 512]), x=x, y=rng.choice(["f32", "bf16"]) if x == "f32" else "bf16",
                    heads=hq + 2 * hkv, rot=hq + hkv, d=d, sx=s, sy=s, sz=d // 2 - 2 * s - rng.choice([0, 0, 1]))
    dtype = rng.choice(["f32", "bf16"])
    d = rng.choice([16, 24, 32, 40, 64, 64, 96, 128])
    hkv = rng.choice([1, 2, 4])
    hq = hkv * rng.choice([1, 1, 2, 4])
    batch = _log_int(rng, 1, 32)
    if kind == "pool":                                  # few query rows against long shapes
        most = min(610000, 40000000 // (hkv * d))
        return dict(kind="attn_fwd", dtype=dtype, batch=batch, n=_log_int(rng, 500, most), queries=rng.choice([1, 1, 1, 3, 16]),
                    hq=hq, hkv=hkv, d=d, keep=rng.choice([1.0, 1.0, 0.75]))
    # attention of all voxels: products of the listed ones' order at most
    pairs = (2.0e11 if dtype == "bf16" else 2.0e10) / (hq * d * (1 if kind == "attn_fwd" else 3))
    most = int(math.sqrt(pairs * batch))                # batch shapes of n / batch rows
    return dict(kind=kind, dtype=dtype, batch=batch, n=_log_int(rng, max(200, 8 * batch), max(400, 16 * batch, min(most, 60000))),
                queries=0, hq=hq, hkv=hkv, d=d, keep=rng.choice([1.0, 1.0, 0.75]))


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------

def _sections(case):
    return [case["sx"], case["sy"], case["sz"]]


def _lengths(case):
    """Voxels of each shape: uneven shares of n, the same for every seed."""
    b, n = case["batch"], case["n"]
    w = [0.4 + math.fmod(0.6180339887 * (i + 1), 1.0) for i in range(b)]
    ls = [max(1, int(n * x / sum(w))) for x in w]
    ls[ls.index(max(ls))] += n - sum(ls)
    return ls


def _offsets(case):
    ko = [0]
    for v in _lengths(case):
        ko.append(ko[-1] + v)
    q = case["queries"]
    return ([q * i for i in range(case["batch"] + 1)] if q else list(ko)), ko


def _inputs(case, seed):
    """The tensors a case's operator takes, on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if kind in ("ln_fwd", "ln_bwd"):
        n, c = case["n"], case["c"]
        x = (normal(n, c) * torch.exp(0.5 * normal(n, 1)) + 0.5 * normal(1, c)).to(DT[case["x"]])   # activations of uneven size
        t = dict(x=x, gamma=1 + 0.2 * normal(c), beta=0.2 * normal(c))
        if kind == "ln_fwd":
            t["r"] = normal(n, c).to(DT[case["x"]]) if case["residual"] else None
        else:
            t["dy"] = normal(n, c).to(DT[case["y"]])
            t["ds"] = normal(n, c).to(DT[case["x"]]) if case["residual"] else None
            m = x.float().mean(1, keepdim=True)
            t["stats"] = torch.cat([m, torch.rsqrt(((x.float() - m) ** 2).mean(1, keepdim=True) + EPS)], 1).contiguous()
        return t
    if kind == "rope":
        n = case["n"]
        return dict(x=normal(n, case["heads"] * case["d"]).to(DT[case["x"]]),
                    pos=torch.randint(0, case["u"], (n, 3), generator=g, device="cuda", dtype=torch.int32))
    hq, hkv, d, dt = case["hq"], case["hkv"], case["d"], DT[case["dtype"]]
    qo, ko = _offsets(case)
    n = case["n"]
    t = {}
    # heads of different sharpness; keys share a direction, as projected features do
    gain = 0.5 + 2.0 * torch.rand(hq, 1, generator=g, device="cuda")
    kk = (normal(n, hkv, d) + 0.5 * normal(1, hkv, d)).reshape(n, hkv * d)
    vv = normal(n, hkv * d)
    qq = (normal(qo[-1], hq, d) * gain).reshape(qo[-1], hq * d)
    if case["queries"]:
        kv = torch.cat([kk, vv], 1).to(dt)
        t.update(q=qq.to(dt), k=kv[:, : hkv * d], v=kv[:, hkv * d:])
    else:                                               # one packed row per voxel, as a projection leaves it
        qkv = torch.cat([qq, kk, vv], 1).to(dt)
        t.update(q=qkv[:, : hq * d], k=qkv[:, hq * d: (hq + hkv) * d], v=qkv[:, (hq + hkv) * d:])
    if kind == "attn_train":
        t["do"] = normal(qo[-1], hq * d).to(dt)
    t["mask"] = None
    if case["keep"] < 1.0:
        m = torch.rand(n, generator=g, device="cuda") < case["keep"]
        if case["batch"] > 2:
            m[ko[1]: ko[2]] = False                     # a shape without any key
        t["mask"] = m.to(torch.uint8)
    return t


def _bytes(nbytes):
    t = torch.empty(int(nbytes) + 256, dtype=torch.uint8, device="cuda")
    off = (-t.data_ptr()) % 256
    return t[off: off + int(nbytes)]


def prepare(case, seed):
    t = _inputs(case, seed)
    state = dict(case=case, t=t)
    kind = case["kind"]
    if kind.startswith("attn"):
        qo, ko = _offsets(case)
        state.update(qo=qo, ko=ko)
    if not own:
        return state
    # what a program that uses the library keeps from step to step: outputs, workspace, offsets
    import paper_1803_11385_amd as hch
    state["hch"] = hch
    new = lambda shape, dt: torch.empty(shape, dtype=DT[dt], device="cuda")
    if kind == "ln_fwd":
        n, c = case["n"], case["c"]
        state.update(y=new((n, c), case["y"]), s=new((n, c), case["x"]) if case["residual"] else None)
    elif kind == "ln_bwd":
        n, c = case["n"], case["c"]
        state.update(dx=new((n, c), case["x"]), dg=new((c,), "f32"), db=new((c,), "f32"),
                     ws=_bytes(hch.hch_layernorm_workspace_bytes(n, c)))
    elif kind == "rope":
        state.update(y=new((case["n"], case["heads"] * case["d"]), case["y"]))
    else:
        b, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
        nq, nk, dt = state["qo"][-1], state["ko"][-1], case["dtype"]
        code = hch.HCH_F32 if dt == "f32" else hch.HCH_BF16
        state["dqo"] = torch.tensor(state["qo"], dtype=torch.int32, device="cuda")
        state["dko"] = state["dqo"] if not case["queries"] else torch.tensor(state["ko"], dtype=torch.int32, device="cuda")
        kinds = [hch.HCH_WS_FWD] + ([hch.HCH_WS_BWD_DATA] if kind == "attn_train" else [])
        state.update(code=code, o=new((nq, hq * d), dt),
                     ws=_bytes(max(hch.hch_attn_workspace_bytes(k, code, b, nq, nk, hq, hkv, d) for k in kinds)))
        if kind == "attn_train":
            g = new((nq, (hq + 2 * hkv) * d), dt)       # gradient of the packed row
            state.update(lse=torch.empty((nq, hq), device="cuda"), dq=g[:, : hq * d], dk=g[:, hq * d: (hq + hkv) * d],
                         dv=g[:, (hq + hkv) * d:])
    return state


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------

def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    hch, case, t = state["hch"], state["case"], state["t"]
    kind = case["kind"]
    code = {"f32": hch.HCH_F32, "bf16": hch.HCH_BF16}
    if kind == "ln_fwd":
        hch.hch_layernorm_fwd(code[case["x"]], t["x"], t["r"], state["s"], t["gamma"], t["beta"], code[case["y"]], state["y"],
                              None, case["n"], case["c"], EPS)
        return [state["s"], state["y"]] if case["residual"] else [state["y"]]
    if kind == "ln_bwd":
        hch.hch_layernorm_bwd(code[case["x"]], t["x"], t["stats"], t["gamma"], code[case["y"]], t["dy"], t["ds"], state["dx"],
                              state["dg"], state["db"], case["n"], case["c"], state["ws"])
        return [state["dx"], state["dg"], state["db"]]
    if kind == "rope":
        f = hch.hch_rope_bwd if case["inverse"] else hch.hch_rope_fwd
        f(code[case["x"]], t["x"], code[case["y"]], state["y"], t["pos"], case["n"], case["heads"], case["rot"], case["d"],
          _sections(case), 10000.0, 1.0)
        return [state["y"]]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    scale = d ** -0.5
    hch.hch_attn_fwd(state["code"], t["q"], t["k"], t["v"], state["o"], state.get("lse"), state["dqo"], state["dko"], t["mask"],
                     hq, hkv, d, scale, state["ws"])
    if kind == "attn_fwd":
        return [state["o"]]
    hch.hch_attn_bwd(state["code"], t["q"], t["k"], t["v"], state["o"], state["lse"], t["do"], state["dq"], state["dk"],
                     state["dv"], state["dqo"], state["dko"], t["mask"], hq, hkv, d, scale, state["ws"])
    return [state["o"], state["dq"], state["dk"], state["dv"]]


def _plain(state):
    case, t = state["case"], state["t"]
    kind = case["kind"]
    if kind == "ln_fwd":
        s = t["x"].float()
        if case["residual"]:
            s = s + t["r"].float()
        m = s.mean(1, keepdim=True)
        z = s - m
        y = z * torch.rsqrt((z * z).mean(1, keepdim=True) + EPS) * t["gamma"] + t["beta"]
        return [s.to(DT[case["x"]]), y.to(DT[case["y"]])] if case["residual"] else [y.to(DT[case["y"]])]
    if kind == "ln_bwd":
        x, dy = t["x"].float(), t["dy"].float()
        rs = t["stats"][:, 1:]
        xh = (x - t["stats"][:, :1]) * rs
        w = dy * t["gamma"]
        dx = rs * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + t["ds"].float()
        return [dx.to(DT[case["x"]]), (dy * xh).sum(0), dy.sum(0)]
    if kind == "rope":
        n, h, d, r = case["n"], case["heads"], case["d"], case["rot"]
        x = t["x"].float().reshape(n, h, d // 2, 2)
        ang = []
        for a, s in enumerate(_sections(case)):
            f = 10000.0 ** (-torch.arange(s, device="cuda", dtype=torch.float32) / max(s, 1))
            ang.append(t["pos"][:, a: a + 1].float() * f)
        ang = torch.cat(ang, 1)[:, None, :]
        if case["inverse"]:
            ang = -ang
        p = ang.shape[2]
        co, si = torch.cos(ang), torch.sin(ang)
        y = x.clone()
        a, b = x[:, :r, :p, 0], x[:, :r, :p, 1]
        y[:, :r, :p, 0] = a * co - b * si
        y[:, :r, :p, 1] = a * si + b * co
        return [y.reshape(n, h * d).to(DT[case["y"]])]
    return _plain_attention(state)


def _plain_attention(state):
    case, t = state["case"], state["t"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group, scale, dt = hq // hkv, d ** -0.5, DT[case["dtype"]]
    train = case["kind"] == "attn_train"
    qo, ko = state["qo"], state["ko"]
    rows = {k: [] for k in ("o", "dq", "dk", "dv")}
    heads = lambda x, h: x.float().reshape(x.shape[0], h, d).transpose(0, 1)              # [h][rows][d]
    back = lambda x: x.transpose(0, 1).reshape(x.shape[1], -1)
    for b in range(case["batch"]):
        sq, sk = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        q = heads(t["q"][sq], hq)
        k, v = (heads(t[x][sk], hkv).repeat_interleave(group, 0) for x in ("k", "v"))
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
        if t["mask"] is not None:
            s = s.masked_fill(t["mask"][sk] == 0, float("-inf"))
        m = s.amax(2, keepdim=True)
        m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
        p = torch.exp(s - m)
        z = p.sum(2, keepdim=True)
        p = p / torch.where(z == 0, torch.ones_like(z), z)                               # no key: a row of zeros
        o = torch.matmul(p, v)
        rows["o"].append(back(o))
        if train:
            do = heads(t["do"][sq], hq)
            dp = torch.matmul(do, v.transpose(1, 2).contiguous())
            ds = p * (dp - (do * o).sum(2, keepdim=True)) * scale
            rows["dq"].append(back(torch.matmul(ds, k)))
            for name, x, y in (("dk", ds, q), ("dv", p, do)):
                w = torch.matmul(x.transpose(1, 2).contiguous(), y)
                rows[name].append(back(w.reshape(hkv, group, -1, d).sum(1)))
    return [torch.cat(rows[k]).to(dt) for k in (("o", "dq", "dk", "dv") if train else ("o",))]


# ---------------------------------------------------------------------------------------------
# cost and truth
# ---------------------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2}
    kind = case["kind"]
    if kind in ("ln_fwd", "ln_bwd"):
        e, r = case["n"] * case["c"], int(case["residual"])
        sx, sy = size[case["x"]], size[case["y"]]
        if kind == "ln_fwd":
            return {"bytes": e * (sx * (1 + 2 * r) + sy) + 8 * case["c"], "flops": (8 + r) * e}
        return {"bytes": e * (sx * (2 + r) + sy) + 8 * case["n"] + 12 * case["c"], "flops": (14 + r) * e}
    if kind == "rope":
        e = case["n"] * case["heads"] * case["d"]
        return {"bytes": e * (size[case["x"]] + size[case["y"]]) + 12 * case["n"],
                "flops": 6 * case["n"] * case["rot"] * sum(_sections(case))}
    qo, ko = _offsets(case)
    pairs = sum((qo[i + 1] - qo[i]) * (ko[i + 1] - ko[i]) for i in range(case["batch"]))
    hq, hkv, d, s = case["hq"], case["hkv"], case["d"], size[case["dtype"]]
    nq, nk = qo[-1], ko[-1]
    f = pairs * case["keep"] * hq * d
    if kind == "attn_fwd":
        return {"bytes": s * d * (2 * nq * hq + 2 * nk * hkv) + (nk if case["keep"] < 1 else 0), "flops": 4 * f}
    return {"bytes": s * d * (4 * nq * hq + 4 * nk * hkv) + (nk if case["keep"] < 1 else 0), "flops": 14 * f}


def exact(case, seed):
    t = {k: (v.double() if v is not None and v.is_floating_point() else v) for k, v in _inputs(case, seed).items()}
    kind = case["kind"]
    if kind == "ln_fwd":
        s = t["x"] + t["r"] if case["residual"] else t["x"]
        y = (s - s.mean(1, keepdim=True)) / torch.sqrt(s.var(1, unbiased=False, keepdim=True) + EPS) * t["gamma"] + t["beta"]
        return [s, y] if case["residual"] else [y]
    if kind == "ln_bwd":
        x, dy, c = t["x"], t["dy"], case["c"]
        mean = x.sum(1, keepdim=True) / c
        sd = torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / c + EPS)
        xh = (x - mean) / sd
        g = dy * t["gamma"]
        dx = (g - g.sum(1, keepdim=True) / c - xh * ((g * xh).sum(1, keepdim=True) / c)) / sd
        if case["residual"]:
            dx = dx + t["ds"]
        return [dx, (xh * dy).sum(0), dy.sum(0)]
    if kind == "rope":
        n, h, d = case["n"], case["heads"], case["d"]
        z = torch.view_as_complex(t["x"].reshape(n, h, d // 2, 2).contiguous()).clone()
        first = 0
        for a, s in enumerate(_sections(case)):
            for j in range(s):
                w = t["pos"][:, a].double() * 10000.0 ** (-j / s)
                turn = torch.polar(torch.ones_like(w), -w if case["inverse"] else w)
                z[:, : case["rot"], first + j] *= turn[:, None]
            first += s
        return [torch.view_as_real(z).reshape(n, h * d)]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    qo, ko = _offsets(case)
    train = kind == "attn_train"
    out = {"o": torch.zeros_like(t["q"])}
    if train:
        out.update(dq=torch.zeros_like(t["q"]), dk=torch.zeros_like(t["k"]), dv=torch.zeros_like(t["v"]))
    for b in range(case["batch"]):
        keys = torch.arange(ko[b], ko[b + 1], device="cuda")
        if t["mask"] is not None:
            keys = keys[t["mask"][keys] != 0]           # only the keys that count
        if keys.numel() == 0:
            continue
        for h in range(hq):
            cq, ck = slice(h * d, h * d + d), slice(h // (hq // hkv) * d, h // (hq // hkv) * d + d)
            k, v = t["k"][keys, ck], t["v"][keys, ck]
            step = max(1, 120000000 // keys.numel())
            for r0 in range(qo[b], qo[b + 1], step):
                r = slice(r0, min(r0 + step, qo[b + 1]))
                s = t["q"][r, cq] @ k.t().contiguous() / math.sqrt(d)
                p = torch.exp(s - torch.logsumexp(s, 1, keepdim=True))
                out["o"][r, cq] = p @ v
                if train:
                    g = t["do"][r, cq]
                    out["dv"][keys, ck] += p.t().contiguous() @ g
                    dp = g @ v.t().contiguous()
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                    out["dq"][r, cq] = ds @ k
                    out["dk"][keys, ck] += ds.t().contiguous() @ t["q"][r, cq]
    return [out[k] for k in (("o", "dq", "dk", "dv") if train else ("o",))]
