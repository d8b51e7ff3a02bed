"""residual_norm and residual_norm_grad against the formulas in 64 bits.

Bounds.  u is half a step of the output's type; e = 2^-24 half a step of fp32.  A row's statistic is
a sum of squares over at most 16 values per lane and then lanes and waves, fewer than 32 additions deep;
its root halves that, and scaling adds a few roundings: 32 e of the terms that a value is made of covers
a forward value, 64 e the first gradient, 128 e the second, which is built on the first.
A sum over `rows` terms in any order is off by at most rows e of the sum of magnitudes."""
import numpy as np
import pytest

from helpers import banner

pytestmark = pytest.mark.gpu

EPS = 1e-5
E = 2.0 ** -24
TYPES = ["f32", "bf16", "f16"]
#        post   gate        scale  pre
PARTS = [(True, "row", True, True), (True, "sequence", True, True), (True, "none", False, True),
         (False, "sequence", True, False), (True, "row", False, False), (False, "none", False, True),
         (False, "none", False, False)]
SHAPES = [(1, 1), (1, 512), (3, 7), (5, 128), (17, 130), (64, 512), (33, 1000), (9, 1024), (300, 200), (7, 2048),
          (5, 2501), (4, 4096), (3, 5000), (2, 8192)]


def _dt(t):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def _half(t):
    import torch
    return torch.finfo(_dt(t)).eps / 2


def _inputs(seed, rows, d, t, post, gate, scale, pre, pad=0, n_seq=5, ld=None, shift=0):
    """CPU tensors; rows `ld` apart and `shift` values off the storage's start."""
    import torch
    g = torch.Generator().manual_seed(seed)
    every = rows + pad

    def rows_of(sigma, n=every):
        wide = torch.zeros(n, (ld or d) + shift)
        wide[:, shift:shift + d] = torch.randn(n, d, generator=g) * sigma
        return wide.to(_dt(t))[:, shift:shift + d]

    s = {"x": rows_of(1.5), "b": rows_of(0.7), "dr": rows_of(0.3), "dn": rows_of(0.2) if pre else None, "rows": rows, "d": d}
    for k, on in (("w_post", post), ("scale", scale), ("w_pre", pre)):
        s[k] = 1.0 + 0.3 * torch.randn(d, generator=g) if on else None
    s["gate"] = s["gate_off"] = None
    if gate == "row":
        s["gate"] = rows_of(1.0)
    if gate == "sequence":
        cut = np.sort(np.random.default_rng(seed).integers(0, rows + 1, n_seq - 1))   # some empty
        s["gate_off"] = torch.tensor(np.concatenate([[0], cut, [rows]]).astype(np.int32))
        s["gate"] = rows_of(1.0, n_seq)
    return s


def _exact(s, r=None):
    """Outputs, gradients and the magnitudes that their bounds go by, in 64 bits; gradients at r."""
    import torch
    D = lambda k: None if s[k] is None else s[k][: s["rows"]].double() if k in ("x", "b", "dr", "dn") else s[k].double()  # noqa: E731
    x, b, dr, dn = D("x"), D("b"), D("dr"), D("dn")
    d = s["d"]
    one = torch.ones(d, dtype=torch.float64)
    w_post, scale, w_pre = [one if s[k] is None else D(k) for k in ("w_post", "scale", "w_pre")]
    if s["gate"] is None:
        gate = one.expand(s["rows"], d)
    elif s["gate_off"] is None:
        gate = s["gate"].double()
    else:
        gate = s["gate"].double().repeat_interleave(torch.diff(s["gate_off"].long()), 0)
    inv = lambda v: 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)  # noqa: E731
    beta = inv(b) if s["w_post"] is not None else torch.ones(s["rows"], 1, dtype=torch.float64)
    add = scale * gate * w_post * b * beta
    o = {"r": x + add}
    size = {"r": x.abs() + add.abs()}
    if s["w_pre"] is not None:
        rho = inv(o["r"])
        o["n"] = w_pre * o["r"] * rho
        size["n"] = 2 * o["n"].abs() + (w_pre * rho).abs() * size["r"]
    at = o["r"] if r is None else r[: s["rows"]].double()
    Dx, Da = dr, dr.abs()
    if s["w_pre"] is not None:
        rho = inv(at)
        Dx = dr + rho * w_pre * dn - at * rho ** 3 * (w_pre * dn * at).mean(1, keepdim=True)
        Da = Da + (rho * w_pre * dn).abs() + at.abs() * rho ** 3 * (w_pre * dn * at).abs().mean(1, keepdim=True)
        o["dw_pre"], size["dw_pre"] = (dn * at * rho).sum(0), (dn * at * rho).abs().sum(0)
    v, va = Dx * scale * gate * w_post, Da * (scale * gate * w_post).abs()
    o["dx"], size["dx"] = Dx, Da
    if s["w_post"] is not None:
        o["db"] = beta * v - b * beta ** 3 * (v * b).mean(1, keepdim=True)
        size["db"] = beta * va + b.abs() * beta ** 3 * (va * b.abs()).mean(1, keepdim=True)
    else:
        o["db"], size["db"] = v, va
    bh = b * beta
    for k, term in (("dw_post", Dx * scale * gate * bh), ("dscale", Dx * gate * w_post * bh)):
        if s[k[1:]] is not None:
            big = Da * (scale * gate * bh).abs() if k == "dw_post" else Da * (gate * w_post * bh).abs()
            o[k], size[k] = term.sum(0), big.sum(0)
    if s["gate"] is not None:
        t, ta = Dx * scale * w_post * bh, Da * (scale * w_post * bh).abs()
        if s["gate_off"] is None:
            o["dgate"], size["dgate"] = t, ta
        else:
            cut = s["gate_off"].tolist()
            o["dgate"] = torch.stack([t[a:e].sum(0) for a, e in zip(cut, cut[1:])])
            size["dgate"] = torch.stack([ta[a:e].sum(0) for a, e in zip(cut, cut[1:])])
    return o, size


def _dev(s):
    """On the GPU with the same strides."""
    def put(v):
        import torch
        if not torch.is_tensor(v):
            return v
        if v.dim() == 2:
            base = torch.empty(0, dtype=v.dtype).set_(v.untyped_storage(), 0, (v.untyped_storage().nbytes() // v.element_size(),))
            return base.cuda().as_strided(v.shape, v.stride(), v.storage_offset())
        return v.cuda()
    return {k: put(v) for k, v in s.items()}


def _params(s):
    return {k: s[k] for k in ("w_post", "gate", "gate_off", "scale", "w_pre")}


def _near(name, got, want, size, u, steps):
    import torch
    got = got.cpu().double()
    assert torch.isfinite(got).all(), name
    over = ((got - want).abs() - (u * want.abs() + steps * E * size)).max().item() if want.numel() else 0.0
    # fp16 results below its normal numbers are off by half of 2^-24
    assert over <= (2.0 ** -25 if u == 2.0 ** -11 else 0.0) + 1e-300, (name, over)


def _check(s, t, out=None):
    from paper_2604_15821_amd import janus
    q, rows = _dev(s), s["rows"]
    r, n = janus.residual_norm(q["x"], q["b"], eps=EPS, **_params(q))
    o, size = _exact(s)
    u = _half(t)
    _near("r", r[:rows], o["r"], size["r"], u, 32)
    assert (n is None) == (s["w_pre"] is None)
    if n is not None:
        _near("n", n[:rows], o["n"], size["n"], u, 32)
    g = janus.residual_norm_grad(q["dr"], q["dn"], r if n is not None else None, q["b"], eps=EPS, **_params(q))
    o, size = _exact(s, r.cpu())
    _near("dx", g.dx[:rows], o["dx"], size["dx"], u, 64)
    _near("db", g.db[:rows], o["db"], size["db"], u, 128)
    for k in ("dw_post", "dscale", "dw_pre"):
        assert (getattr(g, k) is None) == (k not in o), k
        if k in o:
            _near(k, getattr(g, k), o[k], size[k], E, 128 + rows)
    assert (g.dgate is None) == (s["gate"] is None)
    if g.dgate is not None:
        _near("dgate", g.dgate, o["dgate"], size["dgate"], u, 128 + (rows if s["gate_off"] is not None else 0))
    return r, n, g


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,d", SHAPES)
def test_shapes(rows, d, t):
    for k, parts in enumerate(PARTS[:2] if d > 1024 else PARTS):
        banner("residual_norm", rows, d, t, parts)
        _check(_inputs(k + d, rows, d, t, *parts), t)


@pytest.mark.parametrize("rows,d,n_seq", [(5000, 512, 40), (5000, 512, 3), (20_000, 64, 700), (1500, 2048, 9), (2600, 4096, 2),
                                          (4200, 1000, 4200)])
def test_runs_of_rows_and_sequences_across_them(rows, d, n_seq):
    """More rows than groups: sequences within one run, across two and across many; empty ones."""
    banner("residual_norm runs", rows, d, n_seq)
    _check(_inputs(rows, rows, d, "f32" if d < 2048 else "bf16", True, "sequence", True, True, n_seq=n_seq),
           "f32" if d < 2048 else "bf16")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("ld,shift", [(200, 0), (160, 8), (131, 0), (133, 3)])
def test_rows_apart_and_misaligned(t, ld, shift):
    banner("residual_norm strides", t, ld, shift)
    for parts in PARTS[:2]:
        _check(_inputs(ld, 37, 128, t, *parts, ld=ld, shift=shift), t)


def test_rows_behind_the_last_sequence_are_left_alone():
    import torch
    from paper_2604_15821_amd import janus
    banner("residual_norm padding")
    s = _inputs(3, 700, 96, "f32", True, "sequence", True, True, pad=23)
    for k in ("x", "b", "dr", "dn"):
        s[k][700:] = float("nan")   # nothing of them may reach a gradient
    q = _dev(s)
    full = lambda: torch.full((723, 96), 7.0, device="cuda:0")  # noqa: E731
    r, n = janus.residual_norm(q["x"], q["b"], eps=EPS, out=(full(), full()), **_params(q))
    g = janus.residual_norm_grad(q["dr"], q["dn"], r, q["b"], eps=EPS, out=(full(), full()), **_params(q))
    for v in (r, n, g.dx, g.db):
        assert (v[700:] == 7.0).all() and torch.isfinite(v).all()
    o, size = _exact(s, r.cpu())
    _near("dw_pre", g.dw_pre, o["dw_pre"], size["dw_pre"], E, 900)
    _near("dgate", g.dgate, o["dgate"], size["dgate"], E, 900)
    # new outputs are zero there
    r, n = janus.residual_norm(q["x"], q["b"], eps=EPS, **_params(q))
    assert (r[700:] == 0).all() and (n[700:] == 0).all()


@pytest.mark.parametrize("n_seq", [0, 4])
def test_no_rows_and_no_sequences(n_seq):
    """Every row of padding, and no rows at all: outputs untouched, gradients zero."""
    import torch
    from paper_2604_15821_amd import janus
    for rows in (0, 6):
        banner("residual_norm empty", n_seq, rows)
        x = torch.ones(rows, 64, device="cuda:0")
        w = torch.ones(64, device="cuda:0")
        off = torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda:0")
        p = dict(w_post=w, scale=w, w_pre=w, gate=torch.ones(n_seq, 64, device="cuda:0"), gate_off=off)
        r, n = janus.residual_norm(x, x, out=(x.clone(), x.clone()), **p)
        assert (r == 1).all() and (n == 1).all()
        g = janus.residual_norm_grad(x, x, x, x, out=(x.clone(), x.clone()), **p)
        assert (g.dx == 1).all() and (g.db == 1).all() and g.dgate.shape == (n_seq, 64)
        for v in (g.dw_post, g.dscale, g.dw_pre, g.dgate):
            assert (v == 0).all()


def test_in_place():
    import torch
    from paper_2604_15821_amd import janus
    banner("residual_norm in place")
    q = _dev(_inputs(5, 5000, 512, "bf16", True, "row", True, True))
    p = _params(q)
    r, n = janus.residual_norm(q["x"], q["b"], **p)
    x, b = q["x"].clone(), q["b"].clone()
    r2, n2 = janus.residual_norm(x, b, out=(x, b), **p)
    assert torch.equal(r, r2) and torch.equal(n, n2)
    g = janus.residual_norm_grad(q["dr"], q["dn"], r, q["b"], **p)
    dr, dn = q["dr"].clone(), q["dn"].clone()
    h = janus.residual_norm_grad(dr, dn, r, q["b"], out=(dr, dn), **p)
    for a, c in zip(g, h):
        assert torch.equal(a, c)   # and the same on every run


def test_a_row_keeps_its_nan_and_infinity():
    import torch
    from paper_2604_15821_amd import janus
    banner("residual_norm nan")
    q = _dev(_inputs(6, 40, 130, "f32", True, "row", True, True))
    p = _params(q)
    r0, n0 = janus.residual_norm(q["x"], q["b"], **p)
    q["b"][7, 3] = float("nan")
    q["x"][20, 5] = float("inf")
    r, n = janus.residual_norm(q["x"], q["b"], **p)
    keep = [m for m in range(40) if m not in (7, 20)]
    assert torch.equal(r[keep], r0[keep]) and torch.equal(n[keep], n0[keep])
    assert torch.isnan(r[7]).all() and torch.isnan(n[7]).all()
    assert torch.isinf(r[20, 5]) and torch.isnan(n[20, 5])
    z = torch.zeros(3, 64, device="cuda:0")
    w = torch.ones(64, device="cuda:0")
    r, n = janus.residual_norm(z, z, w_post=w, w_pre=w)   # zero rows have a norm through eps
    assert (r == 0).all() and (n == 0).all()


def test_gradient_against_differences():
    """The gradient along a direction against a central difference of the formula in 64 bits."""
    import torch
    from paper_2604_15821_amd import janus
    banner("residual_norm differences")
    s = _inputs(8, 40, 72, "f32", True, "sequence", True, True)
    q = _dev(s)
    r, n = janus.residual_norm(q["x"], q["b"], eps=EPS, **_params(q))
    g = janus.residual_norm_grad(q["dr"], q["dn"], r, q["b"], eps=EPS, **_params(q))
    gen = torch.Generator().manual_seed(1)
    for k, grad in (("x", g.dx), ("b", g.db), ("w_post", g.dw_post), ("gate", g.dgate), ("scale", g.dscale), ("w_pre", g.dw_pre)):
        step = torch.randn(s[k].shape, generator=gen).double()
        loss = []
        for h in (1e-5, -1e-5):
            z = {**s, k: s[k].double() + h * step}
            o, _ = _exact(z)
            loss.append(((o["r"] * s["dr"].double()).sum() + (o["n"] * s["dn"].double()).sum()).item())
        want = (loss[0] - loss[1]) / 2e-5
        size = (grad.cpu().double() * step).abs().sum().item()
        # fp32 gradients of at most 40 rows, and the difference's own curvature (1e-10 of the size)
        assert abs((grad.cpu().double() * step).sum().item() - want) <= (128 + 40) * E * 4 * size + 1e-7 * size, k


def test_missing_dr_is_zero():
    import torch
    from paper_2604_15821_amd import janus
    banner("residual_norm no dr")
    q = _dev(_inputs(9, 50, 256, "f16", True, "row", True, True))
    r, _ = janus.residual_norm(q["x"], q["b"], **_params(q))
    a = janus.residual_norm_grad(None, q["dn"], r, q["b"], **_params(q))
    b = janus.residual_norm_grad(torch.zeros_like(r), q["dn"], r, q["b"], **_params(q))
    for v, w in zip(a, b):
        assert torch.equal(v, w)
