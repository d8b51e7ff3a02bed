"""The expert layer for a few tokens against its formula in 64 bits.

Bounds, with e = 2^-24 and u half a step of the output's type: a pre-activation is a sum of d
products, off by at most (d + 8) e of its magnitudes (matrix instructions may cut off where they round: twice that); SiLU
has a slope below 1.1 and adds (|a| + 16) e of itself; the hidden value enters the second product with at least 16 bits
where the weights have 16 bits (2^-16 of itself); the second product adds (h + 8) e, doubled alike; a gate is off
by twice the error of its logits plus 16 e of itself."""
import numpy as np
import pytest

from helpers import banner

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TYPES = ["f32", "bf16", "f16"]
#         tokens  d    h     n   k  normalize
SHAPES = [(1, 16, 16, 1, 1, False), (1, 64, 128, 4, 1, False), (1, 512, 2048, 64, 2, False), (2, 128, 512, 8, 2, True),
          (3, 48, 80, 5, 5, False), (5, 144, 272, 33, 3, True), (13, 128, 512, 8, 2, False), (16, 96, 64, 3, 2, False),
          (17, 256, 192, 2, 1, False), (31, 64, 64, 256, 8, True), (33, 512, 1040, 7, 4, False), (64, 128, 512, 1, 1, False),
          (64, 208, 336, 16, 8, True), (64, 1024, 512, 130, 6, False), (1, 1600, 48, 200, 4, True), (3, 4112, 32, 253, 8, False)]


def _dt(t):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def _case(seed, tokens, d, h, n, t):
    import torch
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return dict(x=r(tokens, d).to(_dt(t)), router=r(d, n) / d ** 0.5, w_up=(r(n, d, h) / d ** 0.5).to(_dt(t)),
                w_down=(r(n, h, d) / h ** 0.5).to(_dt(t)), beta=0.3 * r(n))


def _check(s, k, normalize, t, got):
    import torch
    y, eid, gate = [v.cpu() for v in got]
    x, router, up, down = [s[q].double() for q in ("x", "router", "w_up", "w_down")]
    d, h = up.shape[1], up.shape[2]
    beta = s["beta"].double() if s["beta"] is not None else torch.zeros(router.shape[1], dtype=torch.float64)
    l = x @ router + beta
    dl = ((d + 8) * 2 * E * (x.abs() @ router.abs() + torch.where(torch.isfinite(beta), beta.abs(), 0.0))).amax(1)
    order = torch.argsort(-l, dim=1, stable=True)[:, :k]
    for m in range(l.shape[0]):   # the choice is decided where logits are further apart than their errors
        top = l[m, order[m]]
        rest = l[m].clone()
        rest[order[m]] = -float("inf")
        gaps = torch.cat([top[:-1] - top[1:], (top[-1:] - rest.max())])
        gaps = gaps[torch.isfinite(gaps)]
        if (gaps > 2 * dl[m]).all():
            assert (eid[m].long() == order[m]).all(), m
        assert len(set(eid[m].tolist())) == k and (eid[m] >= 0).all() and (eid[m] < l.shape[1]).all()
    e = eid.long()
    p = torch.softmax(l, 1).gather(1, e)
    if normalize:
        p = p / p.sum(1, keepdim=True)
    dp = p * (2 * dl[:, None] + 16 * E)
    assert ((gate.double() - p).abs() <= dp).all()
    u = torch.finfo(_dt(t)).eps / 2
    hold = 0.0 if t == "f32" else 2.0 ** -16
    for m in range(x.shape[0]):
        a = torch.stack([x[m] @ up[q] for q in e[m]])
        da = torch.stack([x[m].abs() @ up[q].abs() for q in e[m]]) * (2 * (d + 8) * E)
        v = a * torch.sigmoid(a)
        dv = 1.1 * da + v.abs() * ((a.abs() + 16) * E + hold)
        out = torch.stack([v[c] @ down[q] for c, q in enumerate(e[m])])
        size = torch.stack([v[c].abs() @ down[q].abs() for c, q in enumerate(e[m])])
        dout = torch.stack([dv[c] @ down[q].abs() for c, q in enumerate(e[m])]) + 2 * (h + 8) * E * size
        want = p[m] @ out
        tol = p[m] @ dout + dp[m] @ size + 16 * E * (p[m] @ size)
        tiny = 2.0 ** -25 if t == "f16" else 0.0
        assert ((y[m].double() - want).abs() <= u * want.abs() + tol * (1 + u) + tiny).all(), m


def _run(s, k, normalize=False):
    from paper_2604_15821_amd import janus
    q = {a: None if b is None else b.cuda() for a, b in s.items()}
    return janus.expert_layer(q["x"], q["router"], q["w_up"], q["w_down"], k, beta=q["beta"], normalize=normalize)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,d,h,n,k,normalize", SHAPES)
def test_shapes(tokens, d, h, n, k, normalize, t):
    import torch
    banner("expert_layer", tokens, d, h, n, k, normalize, t)
    s = _case(tokens + d + n, tokens, d, h, n, t)
    if tokens % 2 == 0:
        s["beta"] = None
    got = _run(s, k, normalize)
    _check(s, k, normalize, t, got)
    for a, b in zip(got, _run(s, k, normalize)):
        assert torch.equal(a, b)   # the same on every run


def test_every_token_on_one_expert():
    import torch
    for tokens in (15, 16, 64):
        banner("expert_layer one expert", tokens)
        s = _case(tokens, tokens, 128, 256, 8, "bf16")
        s["beta"] = torch.zeros(8)
        s["beta"][5] = 1000.0
        got = _run(s, 1)
        assert (got[1] == 5).all() and (got[2] == 1).all()
        _check(s, 1, False, "bf16", got)


def test_ties_take_the_lower_index():
    import torch
    banner("expert_layer ties")
    s = _case(1, 6, 64, 64, 70, "f32")
    s["router"][:] = 0.0
    s["beta"] = torch.zeros(70)
    s["beta"][[66, 3, 40]] = 1.0
    got = _run(s, 5)
    assert (got[1].cpu() == torch.tensor([3, 40, 66, 0, 1], dtype=torch.int32)).all()
    _check(s, 5, False, "f32", got)


def test_masked_experts_and_masked_tokens():
    """-inf and the type's lowest value as masks; all experts masked gives zero; fewer left than top_k."""
    import torch
    banner("expert_layer masks")
    s = _case(2, 9, 64, 128, 6, "f32")
    s["beta"] = torch.full((6,), -float("inf"))
    y, eid, gate = _run(s, 2)
    assert (y == 0).all() and (gate == 0).all() and (eid.cpu() == torch.tensor([0, 1], dtype=torch.int32)).all()
    y, eid, gate = _run(s, 2, True)
    assert (y == 0).all() and (gate == 0).all()
    s["beta"][4] = 0.0
    for normalize in (False, True):
        y, eid, gate = _run(s, 2, normalize)
        assert (eid[:, 0] == 4).all() and (gate[:, 0] == 1).all() and (gate[:, 1] == 0).all()
        _check(s, 2, normalize, "f32", (y, eid, gate))
    s["beta"] = torch.full((6,), torch.finfo(torch.float32).min)
    got = _run(s, 2)
    assert torch.isfinite(got[0]).all() and (got[2] == 1 / 6).all()   # x router vanishes next to it
    # a masked expert's weights are not used, also where it fills up the top_k
    s["beta"] = torch.full((6,), -float("inf"))
    s["beta"][4] = 0.0
    clean = _run(s, 3)
    for e in (0, 1, 2, 3, 5):
        s["w_up"][e] = float("nan")
        s["w_down"][e] = float("inf")
    assert torch.equal(_run(s, 3)[0], clean[0])
    s = _case(2, 9, 64, 128, 6, "f32")
    s["beta"] = torch.zeros(6)
    s["beta"][1] = -float("inf")
    s["w_up"][1] = float("nan")
    got = _run(s, 3)
    assert torch.isfinite(got[0]).all()


def test_bad_tokens_stay_alone():
    import torch
    banner("expert_layer nan")
    s = _case(3, 20, 64, 128, 4, "bf16")
    y0, e0, g0 = _run(s, 2)
    s["x"][3, 5] = float("nan")
    s["x"][11, 0] = float("inf")
    y, eid, gate = _run(s, 2)
    keep = [m for m in range(20) if m not in (3, 11)]
    assert torch.equal(y[keep], y0[keep]) and torch.equal(eid[keep], e0[keep]) and torch.equal(gate[keep], g0[keep])
    assert torch.isnan(y[3]).all() and torch.isnan(gate[3]).all() and not torch.isfinite(y[11]).any()
    assert (eid >= 0).all() and (eid < 4).all()


def test_rows_apart_and_no_tokens():
    import torch
    from paper_2604_15821_amd import janus
    banner("expert_layer strides")
    s = _case(4, 7, 64, 96, 4, "f32")
    q = {a: b.cuda() for a, b in s.items()}
    wide = torch.full((7, 200), float("nan"), device="cuda:0")
    wide[:, 8:72] = q["x"]
    out = torch.full((7, 80), 5.0, device="cuda:0")
    got = janus.expert_layer(wide[:, 8:72], q["router"], q["w_up"], q["w_down"], 2, beta=q["beta"], out=out[:, 4:68])
    _check(s, 2, False, "f32", got)
    assert (out[:, :4] == 5).all() and (out[:, 68:] == 5).all()
    y, eid, gate = janus.expert_layer(q["x"][:0], q["router"], q["w_up"], q["w_down"], 2)
    assert y.shape == (0, 64) and eid.shape == (0, 2) and gate.shape == (0, 2)


def test_small_and_large_fp16_weights():
    """Subnormal fp16 weights and hidden values beyond fp16's range take part like others."""
    import torch
    banner("expert_layer fp16 range")
    s = _case(5, 6, 64, 96, 3, "f16")
    s["w_up"] = (s["w_up"].float() * 2.0 ** -20).to(torch.float16)
    s["x"] = (s["x"].float() * 2.0 ** 10).to(torch.float16)
    s["router"] = s["router"] * 2.0 ** -10
    _check(s, 2, False, "f16", _run(s, 2))
    s = _case(6, 6, 64, 96, 3, "f16")
    s["x"] = (s["x"].float() * 2.0 ** 12).to(torch.float16)
    s["w_up"] = (s["w_up"].float() * 2.0 ** 7).to(torch.float16)
    s["w_down"] = (s["w_down"].float() * 2.0 ** -20).to(torch.float16)
    s["router"] = s["router"] * 2.0 ** -12
    got = _run(s, 2)
    assert torch.isfinite(got[0]).all()
    _check(s, 2, False, "f16", got)


def test_more_tokens_on_an_expert_than_planned():
    """A few experts get nearly all tokens, though an even share is a fraction of a tile."""
    import torch
    banner("expert_layer skewed")
    s = _case(7, 61, 96, 160, 40, "f32")
    s["beta"] = torch.zeros(40)
    s["beta"][[4, 30]] = 50.0
    _check(s, 3, False, "f32", _run(s, 3))
