"""Values of the operators around an expert block where few bits or special values show."""
import pytest

from helpers import banner

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _dt(t):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def test_unpacked_silu_far_from_zero():
    """SiLU and SiLU' of stored values from -104 to 104 in fp32.  With e = exp(-|a|): the hardware exponential is good
    to 2 E of itself on [2^-1/2, 2^1/2], where its argument is off by at most 2^-25 (0.4 E of the result), and the
    power of two beside it is exact; at most half of that reaches 1 / (1 + e), whose rounding adds E: 2.2 E for the
    larger of s and 1 - s, and with the error of e and a product 5.6 E for the smaller, 6.6 E for a s.  SiLU' = s (1 + a (1 - s))
    takes 5.6 E of a s (1 - s), and of itself E for the sum, 5.6 E for s and E for either product.  Below fp32's normal
    range a value is off by half a step of 2^-149, |a| times as much where it is multiplied by a."""
    import torch
    from paper_2604_15821_amd import janus
    banner("unpack silu far")
    n = torch.arange(-104, 105, dtype=torch.float64)
    a = torch.cat([n, n / 8, n / 1024, 2.0 ** -torch.arange(1, 100, dtype=torch.float64)])
    a = a[a != 0].reshape(-1, 1)                    # a row each, so each has a scale of its own and is kept exactly
    p = janus.pack_rows(a.float().cuda())
    assert torch.equal(janus.unpack_rows(p, torch.float32).cpu().double(), a)
    g = torch.full_like(a, 0.75).float()
    dx, value = janus.unpack_rows(p, torch.float32, act="silu", grad=g.cuda(), value=True)
    e = torch.exp(-a.abs())
    s, c = torch.where(a > 0, 1 / (1 + e), e / (1 + e)), torch.where(a > 0, e / (1 + e), 1 / (1 + e))
    small = (a.abs() + 2) * 2.0 ** -149
    want, dwant = a * s, g.double() * (s + a * s * c)
    over = ((value.cpu().double() - want).abs() - (7 * E * want.abs() + small)).max().item()
    assert over <= 0, over
    dover = ((dx.cpu().double() - dwant).abs() - 9 * E * dwant.abs() - 6 * E * g.double() * (a * s * c).abs() - small).max().item()
    assert dover <= 0, dover


@pytest.mark.parametrize("tokens", [1, 20])
def test_hidden_silu_far_from_zero(tokens):
    """A hidden value of a large negative pre-activation, taken out by weights of one: 6.6 E for SiLU (see above) and
    nothing for products with one and zero."""
    import torch
    from paper_2604_15821_amd import janus
    banner("expert_layer silu far", tokens)
    x = torch.zeros(tokens, 16)
    x[:, 0] = -20.25 - 3.1875 * torch.arange(tokens)
    if tokens == 1:
        x[0, 0] = -80.8125
    up = torch.zeros(1, 16, 16)
    up[0, 0] = 1.0 + torch.arange(16) / 1024        # a row of pre-activations, products rounded once
    down = torch.eye(16)[None]
    y, _, gate = janus.expert_layer(x.cuda(), torch.zeros(16, 1, device="cuda:0"), up.cuda(), down.cuda(), 1)
    assert (gate == 1).all()
    a = (x[:, :1] * up[0, :1]).double()             # as the kernel rounds the one product
    e = torch.exp(a)
    want = a * e / (1 + e)
    over = ((y.cpu().double() - want).abs() - 7 * E * want.abs() - (a.abs() + 2) * 2.0 ** -149).max().item()
    assert over <= 0, over


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("tokens", [1, 5, 64])
def test_hidden_values_keep_their_bits(tokens, t):
    """Two hidden values near 1, 2^-15 apart, whose difference the second product forms with weights of 1 and -1.
    Pre-activations are exact; a hidden value is off by 3.2 E of itself (positive, see above), its products are exact, and at most six
    additions (three terms of each, zeros add nothing) cut off up to 2 E of the values' sum."""
    import torch
    from paper_2604_15821_amd import janus
    banner("expert_layer hidden bits", tokens, t)
    dt = _dt(t)
    x = torch.zeros(tokens, 16)
    x[:, 0] = 1.3125 + torch.arange(tokens) / 64
    x[:, 1] = 2.0 ** -8
    up = torch.zeros(1, 16, 16)
    up[0, 0, :2] = 1.0
    up[0, 1, 1] = 2.0 ** -7
    down = torch.zeros(1, 16, 16)
    down[0, 0, :] = -1.0
    down[0, 1, :] = 1.0
    x, up, down = x.to(dt), up.to(dt), down.to(dt)
    y, _, gate = janus.expert_layer(x.cuda(), torch.zeros(16, 1, device="cuda:0"), up.cuda(), down.cuda(), 1)
    assert (gate == 1).all()
    h = torch.nn.functional.silu(x.double() @ up[0].double())[:, :2]
    want = (h[:, 1] - h[:, 0])[:, None]
    size = h.sum(1, keepdim=True)
    u = torch.finfo(dt).eps / 2
    tiny = 2.0 ** -25 if t == "f16" else 0.0
    over = ((y.cpu().double() - want).abs() - (u * want.abs() + (4 + 12) * E * size * (1 + u) + tiny)).max().item()
    assert over <= 0, over


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_infinity_in_a_gradient_stays_one(t):
    """G = X^T B with an infinity in B: an infinity of X's sign in its column, NaN where X is zero."""
    import torch
    from paper_2604_15821_amd import janus
    banner("packed_wgrad infinity", t)
    x = torch.randn(90, 40, generator=torch.Generator().manual_seed(1))
    x[30, 7] = x[60, 9] = 0.0
    b = torch.randn(90, 24, generator=torch.Generator().manual_seed(2)).to(_dt(t))
    b[30, 3] = float("inf")
    b[60, 11] = -float("inf")
    b[75, 20] = float("nan")
    p = janus.pack_rows(x.cuda())
    X = janus.unpack_rows(p, torch.float32).cpu().double()
    off = torch.tensor([0, 70, 90], dtype=torch.int32)
    got = janus.packed_wgrad(p, b.cuda(), off.cuda()).cpu()
    want = torch.stack([X[m0:m1].t().contiguous() @ b[m0:m1].double() for m0, m1 in ((0, 70), (70, 90))])
    assert torch.isposinf(want).any() and torch.isneginf(want).any() and torch.isnan(want).any()
    for kind in (torch.isposinf, torch.isneginf, torch.isnan):
        assert torch.equal(kind(got), kind(want))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_finite_activations_come_back_finite(t):
    """A block's rounding can carry the largest values of a type one step beyond it; they come back as its largest
    finite value, and every value within max(max|x| / 127, 2^-127) of its block."""
    import torch
    from paper_2604_15821_amd import janus
    banner("pack_rows top", t)
    dt = _dt(t)
    top = torch.finfo(dt).max
    x = torch.linspace(-1, 1, 96, dtype=torch.float64).repeat(6, 1)
    for m, s in enumerate((1.0, 1 - 2.0 ** -7, 1 - 2.0 ** -6, 0.5, 2.0 ** -8)):
        x[m] *= top * s
    x[5] = top
    x[5, 40] = -top
    x = x.to(dt)
    p = janus.pack_rows(x.cuda())
    size = x.double().abs().view(6, 3, 32).amax(2).repeat_interleave(32, 1)
    for act in ("none", "silu"):
        got = janus.unpack_rows(p, dt, act=act).cpu()
        assert torch.isfinite(got).all()
        if act == "none":
            assert ((got.double() - x.double()).abs() <= (size / 127).clamp(min=2.0 ** -127)).all()
            assert (got[5, :40] == top).all() and got[5, 40] == -top
    g = torch.ones(6, 96, dtype=dt)
    dx, value = janus.unpack_rows(p, dt, act="silu", grad=g.cuda(), value=True)
    assert torch.isfinite(dx).all() and torch.isfinite(value).all()
    x[2, 5] = float("inf")
    got = janus.unpack_rows(janus.pack_rows(x.cuda()), dt).cpu()
    assert torch.isnan(got[2, :32]).all() and torch.isfinite(got[2, 32:]).all()
    wide = torch.tensor([[1e6], [-1e6]], device="cuda:0")      # beyond fp16: as a conversion would have it
    assert torch.equal(janus.unpack_rows(janus.pack_rows(wide), torch.float16).cpu(),
                       torch.tensor([[float("inf")], [-float("inf")]], dtype=torch.float16))


def test_weight_gradient_of_the_most_rows():
    """2^31 - 4097 rows of one column, in one group and in two: every row is in one chunk, and the few that are not
    zero add up exactly."""
    import torch
    from paper_2604_15821_amd import janus
    banner("packed_wgrad most rows")
    rows = 2 ** 31 - 4097
    p = janus.PackedRows(torch.full((rows, 1), 64, dtype=torch.int8, device="cuda:0"),
                         torch.full((rows, 1), 121, dtype=torch.uint8, device="cuda:0"))   # ones
    B = torch.zeros(rows, 1, dtype=torch.bfloat16, device="cuda:0")
    at = [0, 1, 16_223, 16_224, 2 ** 30, 2 ** 30 + 12_345, rows - 16_225, rows - 6, rows - 5, rows - 1]
    for k, m in enumerate(at):
        B[m] = 2.0 ** k
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda:0")
    assert janus.packed_wgrad(p, B, off).item() == 1023
    off = torch.tensor([0, rows - 5, rows], dtype=torch.int32, device="cuda:0")
    assert janus.packed_wgrad(p, B, off).view(-1).tolist() == [255, 768]


def test_the_widest_row():
    """One row of 2^31 - 4097 columns through packing and unpacking."""
    import torch
    from paper_2604_15821_amd import janus
    banner("pack_rows widest")
    d = 2 ** 31 - 4097
    x = torch.zeros(1, d, dtype=torch.bfloat16, device="cuda:0")
    for k, c in enumerate((0, 2047, 2 ** 30 + 5, d - 2049, d - 9, d - 1)):
        x[0, c] = 1.0 + k
    p = janus.pack_rows(x)
    assert p.code.shape == (1, 2 ** 26 - 128) and p.q[0, -1] == 96 and p.code[0, -1] == 123   # 6 = 96 / 16
    assert torch.equal(janus.unpack_rows(p, torch.bfloat16), x)


def test_weight_gradient_of_rows_256_kib_apart():
    """Chunks of 16 224 rows, 262 144 bytes apart: offsets up to the end of 32 bits, the same values as rows side by side."""
    import torch
    from paper_2604_15821_amd import janus
    banner("packed_wgrad far rows")
    rows, P, Q, ld = 33_000, 2048, 4096, 1 << 18
    g = torch.Generator(device="cuda:0").manual_seed(6)
    p = janus.pack_rows(torch.randn(rows, P, generator=g, device="cuda:0"))
    B = torch.randn(rows, Q, generator=g, device="cuda:0").bfloat16()
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda:0")
    q = torch.empty(rows * ld, dtype=torch.int8, device="cuda:0").as_strided((rows, P), (ld, 1))
    q.copy_(p.q)
    assert torch.equal(janus.packed_wgrad(janus.PackedRows(q, p.code), B, off), janus.packed_wgrad(p, B, off))
    far = torch.empty(rows * ld // 2, dtype=torch.bfloat16, device="cuda:0").as_strided((rows, Q), (ld // 2, 1))
    far.copy_(B)
    assert torch.equal(janus.packed_wgrad(p, far, off), janus.packed_wgrad(p, B, off))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_rounding_of_every_block(t):
    """Half a step: at most max|x| / 127 of the block, and 2^-127 where the step is 2^-126 (blocks below 127 2^-126)."""
    import torch
    from paper_2604_15821_amd import janus
    banner("pack_rows bound", t)
    dt = _dt(t)
    low = -149 if t == "f32" else -133 if t == "bf16" else -24
    e = torch.arange(low, 13 if t == "f16" else 125, dtype=torch.float64)
    g = torch.Generator().manual_seed(8)
    x = (torch.rand(len(e), 64, generator=g, dtype=torch.float64) * 2 - 1) * 2.0 ** e[:, None]
    x[:, ::5] = x[:, ::5].sign() * 2.0 ** e[:, None]
    x = x.to(dt)
    p = janus.pack_rows(x.cuda())
    step = (p.code.cpu().double() - 127).exp2().repeat_interleave(32, 1)
    got = p.q.cpu().double() * step
    size = x.double().abs().view(-1, 2, 32).amax(2).repeat_interleave(32, 1)
    assert ((got - x.double()).abs() <= (size / 127).clamp(min=2.0 ** -127)).all()
    if t == "f32":
        assert (got[0] == 0).all() and (size[0] == 2.0 ** -149).all()      # below half of the least step
        assert torch.equal(janus.unpack_rows(p, torch.float32).cpu().double(), got)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens", [1, 20])
def test_infinite_weights_give_what_the_formula_gives(tokens, t):
    """An infinity in W_down gives an infinity of the hidden value's sign in its column, NaN where that is
    zero; one in W_up an infinite hidden value, or NaN where x is zero or its sign the other (-inf times sigmoid(-inf))."""
    import torch
    from paper_2604_15821_amd import janus
    banner("expert_layer infinite weights", tokens, t)
    g = torch.Generator().manual_seed(tokens)
    R = lambda *s: torch.randn(*s, generator=g).to(_dt(t))  # noqa: E731
    c = lambda v: v.cuda()  # noqa: E731
    x, up, down = R(tokens, 32), R(1, 32, 64) / 4, R(1, 64, 48)[:, :, :32].contiguous() / 4
    router = torch.zeros(32, 1)

    def check(up, down):
        y = janus.expert_layer(c(x), c(router), c(up), c(down), 1)[0].cpu()
        a = x.double() @ up[0].double()
        want = (a * torch.sigmoid(a)) @ down[0].double()
        for kind in (torch.isposinf, torch.isneginf, torch.isnan):
            assert torch.equal(kind(y), kind(want))
        return want

    bad = down.clone()
    bad[0, 17, 5], bad[0, 40, 9], bad[0, 3, 30] = float("inf"), -float("inf"), float("nan")
    want = check(up, bad)
    assert torch.isinf(want[:, 5]).all() and torch.isinf(want[:, 9]).all() and torch.isnan(want[:, 30]).all()
    bad = up.clone()
    bad[0, 4, 21] = float("inf")
    check(bad, down)


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_unpacked_silu_next_to_a_rounding_border(t):
    """SiLU and SiLU' of every value that 7 bits and a few powers of two give, in 16 bits: with an fp32 result off by
    1.6 of its steps at most (3.2 E of a s for positive a), only what lies as near to the middle of two 16-bit values may
    be rounded to the other one."""
    import torch
    from paper_2604_15821_amd import janus
    banner("unpack silu borders", t)
    q = torch.arange(1, 128, dtype=torch.int8).repeat(9).reshape(-1, 1)
    code = (127 + torch.arange(-8, 1)).repeat_interleave(127).to(torch.uint8).reshape(-1, 1)
    a = q.double() * (code.double() - 127).exp2()
    want = a / (1 + torch.exp(-a))
    got = janus.unpack_rows(janus.PackedRows(q.cuda(), code.cuda()), _dt(t), act="silu").cpu()
    low, high = (want * (1 - 4 * E)).to(_dt(t)), (want * (1 + 4 * E)).to(_dt(t))
    assert ((got == low) | (got == high)).all()
    assert (got == want.to(_dt(t))).double().mean() > 0.998
    if t == "bf16":
        near = (a == 5.9375).nonzero()[0, 0]
        assert got[near] == want[near].to(_dt(t))      # 1.18 fp32 steps below the middle
