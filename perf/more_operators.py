"""More operators whose speed is measured, beside their plain forms.

* ``norm``       the residual's addition and an RMS norm (``add_rms_norm``);
                 ``norm_i8`` with the norm's output in 8 bits, a scale for each
                 row (``add_rms_norm_i8``); ``norm_bwd`` the gradients
                 (``add_rms_norm_backward``)
* ``adapt``      a linear layer shared by a packed batch of requests, each with
                 the low-rank adapter of its own (``adapter_linear``);
                 ``adapt_step`` a training step of the adapters, forward and
                 backward (``adapter_linear_backward``)
* ``adamw``      an AdamW step over many tensors at once (``AdamW``)

With ``own`` false ``run`` computes them from elementary torch operations in
fp32 (fp64 where a value may sit on a rounding border or a sum is long),
rounded once at the end; with ``own`` true it calls the package.
"""
import math

import torch

own = False

DEV = "cuda"
F32, F64 = torch.float32, torch.float64


def listed():
    return [
        # one token's row before a layer: nothing but latency
        dict(name="norm_one_row", kind="norm", dtype="bf16", resid="same", rows=1, K=4096),
        # a packed batch of several tenants' images, the residual stream in fp32
        dict(name="norm_packed", kind="norm", dtype="bf16", resid="f32", rows=7531, K=1152),
        # a small batch of an odd width on its way into an 8-bit layer
        dict(name="norm_i8_odd", kind="norm_i8", dtype="bf16", resid="same", rows=333, K=1051),
        # a wide model's 1024-px image with guidance before its 8-bit projections
        dict(name="norm_i8_wide", kind="norm_i8", dtype="bf16", resid="same", rows=8192, K=4096),
        # gradients for a ragged batch of small images, the stream in fp32
        dict(name="norm_bwd_ragged", kind="norm_bwd", dtype="bf16", resid="f32", rows=4451, K=1152),
        # gradients of a very wide layer's norm
        dict(name="norm_bwd_wide", kind="norm_bwd", dtype="bf16", resid="same", rows=4096, K=10240),
        # single tokens of 24 requests with 16 tenants' adapters between them
        dict(name="adapt_tokens", kind="adapt", dtype="bf16", M=24, N=4096, K=4096, n=16, r=16,
             order="scattered", bias=False),
        # a packed batch of 8 requests, some of which have no adapter
        dict(name="adapt_packed", kind="adapt", dtype="bf16", M=7531, N=4608, K=1152, n=8, r=32,
             order="runs", bias=True),
        # an adapter's training in fp32, as a check of bf16 results is run; no size a multiple of anything
        dict(name="adapt_step_odd", kind="adapt_step", dtype="f32", M=333, N=1155, K=1153, n=2, r=5,
             order="runs", bias=True),
        # four tenants' adapters of a wide layer trained at once
        dict(name="adapt_step_wide", kind="adapt_step", dtype="bf16", M=4096, N=4096, K=4096, n=4, r=16,
             order="runs", bias=False),
        # the adapters of two projections in each of 28 blocks
        dict(name="adamw_adapters", kind="adamw", dtype="f32", layers=56, a=16, b=1152),
        # the MLP weights of four blocks, kept in bf16 beside fp32 masters
        dict(name="adamw_layers", kind="adamw", dtype="bf16", layers=4, a=1152, b=4608),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_i8", "norm_bwd", "adapt", "adapt_step", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind.startswith("norm"):
        K, rows = _log(rng, 16, 16384), _log(rng, 1, 32768)
        if rng.random() < 0.5:
            K = (K + 7) // 8 * 8
        rows = max(1, min(rows, 4096 * 10240 // (2 * K)))
        resid = "same" if dtype == "f32" else rng.choice(["same", "f32"])
        if kind != "norm_bwd" and rng.random() < 0.2:
            resid = "none"
        return dict(kind=kind, dtype=dtype, resid=resid, rows=rows, K=K)
    if kind in ("adapt", "adapt_step"):
        # bf16 rows are loaded in whole 16-byte pieces: widths in eights
        M, N, K = _log(rng, 1, 8192), 8 * _log(rng, 8, 1024), 8 * _log(rng, 8, 1024)
        r, n = rng.choice([4, 8, 16, 32, 64, _log(rng, 1, 64)]), rng.choice([1, 2, 4, 8, 16, 32])
        n = min(n, 512 // r)
        cap = 4096 * 4096 * 4096 if dtype == "bf16" else 4096 * 4096 * 4096 // 16
        if kind == "adapt_step":
            cap //= 3
        M = max(1, min(M, cap // (N * K)))
        if dtype == "f32":
            N += rng.choice([0, 1, 3])
            K += rng.choice([0, 1, 3])
        return dict(kind=kind, dtype=dtype, M=M, N=N, K=K, n=n, r=r, order=rng.choice(["runs", "runs", "scattered"]),
                    bias=rng.random() < 0.5)
    a, b = _log(rng, 4, 1152), _log(rng, 64, 4608)
    layers = max(1, min(_log(rng, 1, 120), 4 * 1152 * 4608 // (a * b)))
    return dict(kind=kind, dtype=dtype, layers=layers, a=a, b=b)


# ------------------------------------------------------------------ inputs

EPS = 1e-6
ADAMW = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _index(g, case):
    """The adapter of every row, -1: none.  ``runs``: requests of random lengths one after
    the other, an eighth of them without an adapter; ``scattered``: a row each."""
    M, n = case["M"], case["n"]
    if case["order"] == "scattered":
        return torch.randint(-1 if n > 1 else 0, n, (M,), generator=g, device=DEV, dtype=torch.int32)
    ends = torch.rand(2 * n - 1, generator=g, device=DEV).sort().values * M
    request = torch.searchsorted(ends, torch.arange(M, device=DEV, dtype=F32) + 0.5, right=True)
    taken = torch.randperm(2 * n, generator=g, device=DEV) % n
    without = torch.rand(2 * n, generator=g, device=DEV) < 0.125
    return torch.where(without, torch.full_like(taken, -1), taken)[request].to(torch.int32)


def _stacks(case):
    """Shapes of the weights of one kind, all layers in one buffer"""
    L, a, b = case["layers"], case["a"], case["b"]
    return [(L, a, b), (L, b, a), (L, b)]


def _each(stacks):
    """The single weights: views of the stacks, layer by layer"""
    return [s[i] for i in range(stacks[0].shape[0]) for s in stacks]


def _inputs(case, seed):
    g, dt, kind = _gen(seed), _dt(case), case["kind"]
    if kind.startswith("norm"):
        rows, K = case["rows"], case["K"]
        rt = F32 if case["resid"] == "f32" else dt
        st = dict(w=(1 + _randn(g, (K,), 0.2, F32)).to(dt), resid=None)
        # a few features far larger than the rest, as a stream has them
        big = 1 + 12 * (torch.rand(K, generator=g, device=DEV) < 0.01).to(F32)
        if kind == "norm_bwd":
            st.update(h=(_randn(g, (rows, K), 2.0, F32) * big).to(rt), dy=_randn(g, (rows, K), 1.0, dt),
                      dh=_randn(g, (rows, K), 1.0, rt))
        else:
            st.update(x=_randn(g, (rows, K), 1.0, dt))
            if case["resid"] != "none":
                st.update(resid=(_randn(g, (rows, K), 2.0, F32) * big).to(rt))
        return st
    if kind in ("adapt", "adapt_step"):
        M, N, K, n, r = (case[k] for k in ("M", "N", "K", "n", "r"))
        st = dict(x=_randn(g, (M, K), 1.0, dt), w=_randn(g, (N, K), K ** -0.5, dt),
                  a=_randn(g, (n, r, K), K ** -0.5, dt), b=_randn(g, (n, N, r), 0.3 * r ** -0.5, dt),
                  scale=0.5 + 1.5 * torch.rand(n, generator=g, device=DEV), index=_index(g, case),
                  bias=_randn(g, (N,), 0.1, dt) if case["bias"] else None)
        if kind == "adapt_step":
            st.update(dy=_randn(g, (M, N), 1.0, dt))
        return st
    # some steps into a training: moments of the gradients' size
    shapes = _stacks(case)
    st = dict(p=[_randn(g, s, 0.05, F32) for s in shapes], m=[_randn(g, s, 0.003, F32) for s in shapes],
              v=[_randn(g, s, 0.01, F32).square() for s in shapes], step=7,
              # gradients as backward passes leave them, a tensor each
              g=[t.clone() for t in _each([_randn(g, s, 0.01, dt) for s in shapes])])
    if dt != F32:
        st.update(low=[p.to(dt) for p in st["p"]])
    return st


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if case["kind"] == "adamw" and own:
        import paper_2607_26566_amd as t2i
        # the optimizer that a training program keeps beside its weights
        masters = dict(masters=_each(st["p"])) if "low" in st else {}
        st["opt"] = t2i.AdamW(_each(st.get("low", st["p"])), exp_avg=_each(st["m"]), exp_avg_sq=_each(st["v"]),
                              step=st["step"], **masters, **ADAMW)
    return st


# ------------------------------------------------------------------ plain forms

def _plain_sum(st):
    """h in its own type"""
    return st["x"] if st["resid"] is None else (st["resid"].to(F32) + st["x"].to(F32)).to(st["resid"].dtype)


def _rstd(h):
    return torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)


def _plain_norm(st):
    h = _plain_sum(st)
    h32 = h.to(F32)
    return dict(y=(h32 * _rstd(h32) * st["w"].to(F32)).to(st["x"].dtype), h=h)


def _plain_norm_i8(st):
    h = _plain_sum(st)
    t = h.to(F64) * st["w"].to(F64)     # fp64: a quotient may lie next to a half
    top = t.abs().amax(-1, keepdim=True)
    q = torch.round(127 * t / torch.where(top > 0, top, torch.ones_like(top))).to(F32)
    return dict(v=q * (top.to(F32) * _rstd(h.to(F32)) / 127), h=h)


def _plain_norm_bwd(st):
    h, w = st["h"].to(F32), st["w"].to(F32)
    dy = st["dy"].to(F32)
    r = _rstd(h)
    n = h * r
    d = dy * w
    dsum = st["dh"].to(F32) + r * (d - n * (d * n).mean(-1, keepdim=True))
    return dict(dx=dsum.to(st["dy"].dtype), dresid=dsum.to(st["h"].dtype),
                dw=(dy * n).to(F64).sum(0).to(st["w"].dtype))


def _chosen(st):
    """[M, n, 1] of the scale where a row takes an adapter, else 0"""
    n = st["a"].shape[0]
    took = st["index"][:, None] == torch.arange(n, device=DEV)[None]
    return (took.to(F32) * st["scale"])[..., None]


def _wide(st):
    """all adapters side by side: [n r, K] and [N, n r]"""
    return st["a"].to(F32).flatten(0, 1), st["b"].to(F32).permute(1, 0, 2).flatten(1)


def _plain_adapt(st):
    x, (a, b), c = st["x"].to(F32), _wide(st), _chosen(st)
    t = ((x @ a.T).unflatten(1, (c.shape[1], -1)) * c).flatten(1)
    y = x @ st["w"].to(F32).T + t @ b.T
    if st["bias"] is not None:
        y = y + st["bias"].to(F32)
    return y, t, a, b, c


def _plain_adapt_step(st):
    y, t, a, b, c = _plain_adapt(st)
    n, r, K = st["a"].shape
    dy, x = st["dy"].to(F32), st["x"].to(F32)
    u = ((dy @ b).unflatten(1, (n, r)) * c).flatten(1)
    out = dict(y=y, dx=dy @ st["w"].to(F32) + u @ a, da=(u.T @ x).view(n, r, K),
               db=(dy.T @ t).unflatten(1, (n, r)).permute(1, 0, 2))
    return {k: v.to(st["x"].dtype).contiguous() for k, v in out.items()}


def _plain_adamw_stack(p, g, m, v, step):
    b1, b2 = ADAMW["betas"]
    g = torch.stack(g).to(F32)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    mh, vh = m / (1 - b1 ** step), v / (1 - b2 ** step)
    return p - ADAMW["lr"] * (mh / (vh.sqrt() + ADAMW["eps"]) + ADAMW["weight_decay"] * p), m, v


def _plain_adamw(st):
    st["step"] += 1
    new = [_plain_adamw_stack(st["p"][i], st["g"][i::3], st["m"][i], st["v"][i], st["step"]) for i in range(3)]
    st.update(zip("pmv", map(list, zip(*new))))
    if "low" in st:
        st["low"] = [p.to(st["low"][0].dtype) for p in st["p"]]


def _results(st):
    """The updated weights and state"""
    return {k: st[k] for k in ("p", "m", "v", "low") if k in st}


# ------------------------------------------------------------------ one pass

def run(st):
    c, kind = st["case"], st["case"]["kind"]
    if not own:
        if kind == "adapt":
            return _plain_adapt(st)[0].to(_dt(c))
        if kind == "adamw":
            _plain_adamw(st)
            return _results(st)
        return dict(norm=_plain_norm, norm_i8=_plain_norm_i8, norm_bwd=_plain_norm_bwd,
                    adapt_step=_plain_adapt_step)[kind](st)
    import paper_2607_26566_amd as t2i
    if kind == "norm":
        y, h = t2i.add_rms_norm(st["x"], st["w"], st["resid"], eps=EPS)
        return dict(y=y, h=h)
    if kind == "norm_i8":
        q, s, h = t2i.add_rms_norm_i8(st["x"], st["w"], st["resid"], eps=EPS)
        return dict(v=q[:, :c["K"]] * s[:, None], h=h)
    if kind == "norm_bwd":
        dx, dresid, dw = t2i.add_rms_norm_backward(st["dy"], st["h"], st["w"], st["dh"], eps=EPS)
        return dict(dx=dx, dresid=dx if dresid is None else dresid, dw=dw)
    ad = dict(index=st.get("index"), scale=st.get("scale"))
    if kind == "adapt":
        return t2i.adapter_linear(st["x"], st["w"], st["a"], st["b"], st["bias"], **ad)
    if kind == "adapt_step":
        y, t = t2i.adapter_linear(st["x"], st["w"], st["a"], st["b"], st["bias"], save_t=True, **ad)
        dx, da, db = t2i.adapter_linear_backward(st["dy"], st["x"], st["w"], st["a"], st["b"], t, **ad)
        return dict(y=y, dx=dx, da=da, db=db)
    st["opt"].step(st["g"])
    return _results(st)


def work(case):
    kind, e = case["kind"], 4 if case["dtype"] == "f32" else 2
    if kind.startswith("norm"):
        rows, K = case["rows"], case["K"]
        re = 4 if case["resid"] == "f32" else e
        if kind == "norm_bwd":   # dy, h, dh in; the sum's gradient out in the types of both operands
            return dict(bytes=rows * K * (2 * e + 3 * re - (e if re == e else 0)) + 2 * e * K, flops=12 * rows * K)
        out = rows * (K + 4) if kind == "norm_i8" else e * rows * K
        return dict(bytes=rows * K * (e + (0 if case["resid"] == "none" else 2 * re)) + e * K + out,
                    flops=6 * rows * K)
    if kind in ("adapt", "adapt_step"):
        M, N, K, n, r = (case[k] for k in ("M", "N", "K", "n", "r"))
        some = min(n, M)   # adapters that rows take, at most
        ad = some * r * (N + K)
        fwd = M * K + N * K + ad + M * N + N * case["bias"]
        if kind == "adapt":
            return dict(bytes=e * fwd + 4 * M + 4 * n, flops=2 * M * N * K + 2 * M * r * (N + K))
        # dy in; the gradients of x and of all adapters out
        return dict(bytes=e * (fwd + M * N + M * K + n * r * (N + K)) + 4 * M + 4 * n,
                    flops=4 * M * N * K + 6 * M * r * (N + K))
    count = sum(math.prod(s) for s in _stacks(case))
    return dict(bytes=count * (24 + e + (0 if e == 4 else 2)), flops=14 * count)


# ------------------------------------------------------------------ float64, from the definitions

def _e_norm(h, w):
    return h / torch.sqrt(h.pow(2).sum(-1, keepdim=True) / h.shape[-1] + EPS) * w


def _e_adapters(st, x):
    """For every adapter: the rows that take it, and its two matrices, the scale in the first"""
    for i in range(st["a"].shape[0]):
        rows = torch.nonzero(st["index"] == i)[:, 0]
        yield i, rows, x[rows], st["scale"][i].to(F64) * st["a"][i].to(F64), st["b"][i].to(F64)


def exact(case, seed):
    st, kind = _inputs(case, seed), case["kind"]
    if kind in ("norm", "norm_i8"):
        h = st["x"].to(F64)
        if st["resid"] is not None:   # (h is a value of the stream's type)
            h = (h + st["resid"].to(F64)).to(st["resid"].dtype).to(F64)
        w = st["w"].to(F64)
        if kind == "norm":
            return dict(y=_e_norm(h, w), h=h)
        # a value's code does not depend on the norm's factor, which its row has in common
        most = (h * w).abs().max(-1, keepdim=True).values
        size = _e_norm(h, w).abs().max(-1, keepdim=True).values
        return dict(v=torch.round(h * w * 127 / most) * size / 127, h=h)
    if kind == "norm_bwd":
        with torch.enable_grad():
            h, w = st["h"].to(F64).requires_grad_(), st["w"].to(F64).requires_grad_()
            dx, dw = torch.autograd.grad(_e_norm(h, w), (h, w), st["dy"].to(F64))
        dx = dx + st["dh"].to(F64)
        return dict(dx=dx, dresid=dx, dw=dw)
    if kind in ("adapt", "adapt_step"):
        x = st["x"].to(F64)
        w = st["w"].to(F64)
        y = torch.mm(x, w.t())
        if st["bias"] is not None:
            y += st["bias"].to(F64)
        for _, rows, xr, a, b in _e_adapters(st, x):
            y[rows] += torch.mm(torch.mm(xr, a.t()), b.t())
        if kind == "adapt":
            return y
        dy = st["dy"].to(F64)
        dx = torch.mm(dy, w)
        da, db = torch.zeros_like(st["a"], dtype=F64), torch.zeros_like(st["b"], dtype=F64)
        for i, rows, xr, a, b in _e_adapters(st, x):
            back = torch.mm(dy[rows], b)
            dx[rows] += torch.mm(back, a)
            da[i] = st["scale"][i].to(F64) * torch.mm(back.t(), xr)
            db[i] = torch.mm(dy[rows].t(), torch.mm(xr, a.t()))
        return dict(y=y, dx=dx, da=da, db=db)
    (b1, b2), t = ADAMW["betas"], st["step"] + 1
    new = dict(p=[], m=[], v=[])
    for i, (p, m, v) in enumerate(zip(*([x.to(F64) for x in st[k]] for k in "pmv"))):
        g = torch.stack([x.to(F64) for x in st["g"][i::3]])
        m = m + (g - m) * (1 - b1)
        v = v + (g.pow(2) - v) * (1 - b2)
        way = m / (1 - b1 ** t) / (torch.sqrt(v / (1 - b2 ** t)) + ADAMW["eps"])
        new["p"].append(p * (1 - ADAMW["lr"] * ADAMW["weight_decay"]) - ADAMW["lr"] * way)
        new["m"].append(m)
        new["v"].append(v)
    if "low" in st:
        new["low"] = new["p"]
    return _results(new)
