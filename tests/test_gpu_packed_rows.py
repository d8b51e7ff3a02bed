"""Activations in 8 bits: packing and unpacking value by value, and the weight gradient that reads them
against the sums in 64 bits."""
import numpy as np
import pytest

from helpers import banner

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TYPES = ["f32", "bf16", "f16"]
SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (7, 64), (5, 100), (129, 200), (64, 512), (3, 1024), (5, 2048), (2, 4100),
          (70_000, 40)]


def _dt(t):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def _pack_exact(x):
    """(q, code) of x [rows, d] by the definition, in 64 bits on the CPU."""
    x = x.astype(np.float64)
    rows, d = x.shape
    q = np.zeros((rows, d), np.int8)
    code = np.zeros((rows, (d + 31) // 32), np.uint8)
    for j in range(code.shape[1]):
        v = x[:, 32 * j:32 * j + 32]
        top = np.abs(v).max(1)
        fine = np.isfinite(v).all(1)
        e = np.full(rows, -126)
        with np.errstate(invalid="ignore"):
            for _ in range(260):
                e = np.where(fine & (np.where(fine, top, 0) > 127.0 * 2.0 ** e.astype(float)), e + 1, e)
        code[:, j] = np.where(fine, e + 127, 255)
        n = np.rint(np.where(fine[:, None], v, 0) / 2.0 ** e.astype(float)[:, None])
        q[:, 32 * j:32 * j + 32] = np.where(fine[:, None], n, 0)
    return q, code


def _values(q, code):
    step = np.where(code == 255, np.nan, 2.0 ** (code.astype(np.float64) - 127))
    return q.astype(np.float64) * np.repeat(step, 32, 1)[:, :q.shape[1]]


def _x(seed, rows, d, t, spread=3.0):
    """Values over many magnitudes, blocks of zeros, borders of the scale rule, ties."""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, d)) * 2.0 ** rng.uniform(-spread, spread, (rows, 1))
    x[rng.random((rows, d)) < 0.05] = 0.0
    if rows > 2:
        x[0] = 0.0
        x[1] = 127.0                                  # the largest of its scale
        x[2] = np.where(np.arange(d) % 2, 127.5, 1.5)   # the next scale, ties
    return torch.from_numpy(x).to(_dt(t))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,d", SHAPES)
def test_pack_and_unpack_are_exact(rows, d, t):
    import torch
    from paper_2604_15821_amd import janus
    banner("pack_rows", rows, d, t)
    x = _x(rows + d, rows, d, t)
    p = janus.pack_rows(x.cuda())
    q, code = _pack_exact(x.float().numpy())
    assert (p.q.cpu().numpy() == q).all() and (p.code.cpu().numpy() == code).all()
    want = torch.from_numpy(_values(q, code))
    assert (want - x.double()).abs().max() <= x.double().abs().max() / 127
    for out in TYPES:
        got = janus.unpack_rows(p, _dt(out))
        assert torch.equal(got.cpu(), want.to(_dt(out)))
        into = torch.empty_like(got)
        assert janus.unpack_rows(p, _dt(out), out=into) is into and torch.equal(into, got)


def test_pack_keeps_strides_and_the_columns_between():
    import torch
    from paper_2604_15821_amd import janus
    for ldx, ldq, shift in ((57, 57, 0), (64, 72, 8), (61, 80, 3)):
        banner("pack_rows strides", ldx, ldq, shift)
        x = _x(4, 33, 50, "bf16")
        wide = torch.full((33, ldx + shift), float("inf"), dtype=torch.bfloat16, device="cuda:0")
        wide[:, shift:shift + 50] = x.cuda()
        q = torch.full((33, ldq + shift), 77, dtype=torch.int8, device="cuda:0")
        code = torch.full((33, 5), 99, dtype=torch.uint8, device="cuda:0")
        p = janus.pack_rows(wide[:, shift:shift + 50], out=janus.PackedRows(q[:, shift:shift + 50], code[:, 1:3]))
        want_q, want_code = _pack_exact(x.float().numpy())
        assert (p.q.cpu().numpy() == want_q).all() and (p.code.cpu().numpy() == want_code).all()
        assert (q[:, :shift] == 77).all() and (q[:, shift + 50:] == 77).all()
        assert (code[:, 0] == 99).all() and (code[:, 3:] == 99).all()
        got = janus.unpack_rows(p, torch.float32)
        assert (got.cpu().numpy() == _values(want_q, want_code)).all()


def test_pack_extremes():
    """Infinities and NaN take their own block only; the smallest and largest magnitudes."""
    import torch
    from paper_2604_15821_amd import janus
    banner("pack_rows extremes")
    x = torch.ones(6, 96)
    x[0, 40] = float("nan")
    x[1, 5] = float("-inf")
    x[2, :] = torch.finfo(torch.float32).max
    x[3, :] = 2.0 ** -149
    x[4, :32] = 2.0 ** -126 * 0.5
    x[5, 64:] = -torch.finfo(torch.float32).max
    p = janus.pack_rows(x.cuda())
    q, code = _pack_exact(x.numpy())
    assert (p.q.cpu().numpy() == q).all() and (p.code.cpu().numpy() == code).all()
    got = janus.unpack_rows(p, torch.float32).cpu()
    bad = torch.zeros(6, 96, dtype=torch.bool)
    bad[0, 32:64] = bad[1, :32] = True
    assert (torch.isnan(got) == bad).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (5, 100), (129, 200), (64, 512), (3, 2048)])
def test_silu_and_its_gradient(rows, d, t):
    """s = 1 / (1 + exp(-a)) is good to (|a| + 16) e of itself: the exponent a log2(e) is rounded (|a| e in
    the result), then exponential, sum and reciprocal.  SiLU' = s + a s (1 - s), where 1 - s is off by the
    error of s."""
    import torch
    from paper_2604_15821_amd import janus
    banner("unpack silu", rows, d, t)
    p = janus.pack_rows(_x(d, rows, d, "f32").cuda())
    a = torch.from_numpy(_values(p.q.cpu().numpy(), p.code.cpu().numpy()))
    g = torch.randn(rows, d, generator=torch.Generator().manual_seed(1)).to(_dt(t))
    u = torch.finfo(_dt(t)).eps / 2
    tiny = torch.finfo(_dt(t)).smallest_normal * u
    s = torch.sigmoid(a)
    err = (a.abs() + 16) * E
    want, size = a * s, (a * s).abs() * err
    dwant = g.double() * (s + a * s * (1 - s))
    dsize = g.double().abs() * (s * (err + 8 * E) + a.abs() * s * ((1 - s) * (err + 8 * E) + s * err + E))
    dx, value = janus.unpack_rows(p, _dt(t), act="silu", grad=g.cuda(), value=True)
    assert ((value.cpu().double() - want).abs() <= u * want.abs() + size * (1 + u) + tiny).all()
    assert ((dx.cpu().double() - dwant).abs() <= u * dwant.abs() + dsize * (1 + u) + tiny).all()
    assert torch.equal(janus.unpack_rows(p, _dt(t), act="silu"), value)
    mine = g.cuda()
    assert torch.equal(janus.unpack_rows(p, _dt(t), act="silu", grad=mine, out=mine), dx) and torch.equal(mine, dx)


def _wgrad_case(seed, sizes, P, Q, t, pad=0):
    import torch
    rows = int(sum(sizes)) + pad
    x = _x(seed, rows, P, "f32")
    b = torch.randn(rows, Q, generator=torch.Generator().manual_seed(seed)).to(_dt(t))
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32))
    return x, b, off


def _wgrad_check(p, b, off, G, t):
    """Products are exact, so only additions round: at most 3 per row (an fp32 value goes in as three terms),
    each to a whole step (2 e) where the matrix unit cuts off, plus the joins of the chunks."""
    import torch
    X = torch.from_numpy(_values(p.q.cpu().numpy(), p.code.cpu().numpy()))
    G = G.cpu().double()
    terms = {"bf16": 1, "f16": 2, "f32": 3}[t]
    for g, (m0, m1) in enumerate(zip(off.tolist(), off.tolist()[1:])):
        want = X[m0:m1].t() @ b[m0:m1].double()
        size = X[m0:m1].abs().t() @ b[m0:m1].double().abs()
        over = ((G[g] - want).abs() - (2 * terms * (m1 - m0) + 64) * E * size).max().item()
        assert over <= 0.0, (g, over)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("sizes,P,Q", [([1], 1, 1), ([0, 3, 0], 5, 9), ([16, 17, 1], 33, 40), ([100], 64, 64),
                                       ([63, 65, 0, 2], 130, 72), ([700, 0, 1300, 129], 128, 512), ([300], 200, 260),
                                       ([40, 41], 16, 1000), ([2000, 31], 520, 24), ([9], 257, 129)])
def test_wgrad(sizes, P, Q, t):
    from paper_2604_15821_amd import janus
    banner("packed_wgrad", sizes, P, Q, t)
    x, b, off = _wgrad_case(P + Q, sizes, P, Q, t)
    p = janus.pack_rows(x.cuda())
    G = janus.packed_wgrad(p, b.cuda(), off.cuda())
    _wgrad_check(p, b, off, G, t)


@pytest.mark.parametrize("groups", [64, 65, 300, 1024])
def test_wgrad_many_groups(groups):
    """Some groups are empty, and one is long enough for several chunks."""
    import numpy as np
    from paper_2604_15821_amd import janus
    banner("packed_wgrad groups", groups)
    sizes = np.random.default_rng(groups).integers(0, 20, groups)
    sizes[groups // 3] = 2500
    x, b, off = _wgrad_case(groups, sizes.tolist(), 24, 16, "bf16")
    p = janus.pack_rows(x.cuda())
    _wgrad_check(p, b, off, janus.packed_wgrad(p, b.cuda(), off.cuda()), "bf16")


@pytest.mark.parametrize("t", TYPES)
def test_wgrad_many_chunks_of_odd_blocks(t):
    """Groups of 18 and of 2 chunks whose gradients are no multiple of four values."""
    from paper_2604_15821_amd import janus
    banner("packed_wgrad odd blocks", t)
    x, b, off = _wgrad_case(11, [9000, 700, 1], 33, 37, t)
    p = janus.pack_rows(x.cuda())
    _wgrad_check(p, b, off, janus.packed_wgrad(p, b.cuda(), off.cuda()), t)


@pytest.mark.parametrize("rows,P,Q", [(9000, 300, 520), (4000, 1024, 1030), (1200, 2048, 64)])
def test_wgrad_one_group(rows, P, Q):
    """Fewer chunks than dies, with many tiles each."""
    from paper_2604_15821_amd import janus
    banner("packed_wgrad one group", rows, P, Q)
    x, b, off = _wgrad_case(rows, [rows], P, Q, "f16")
    p = janus.pack_rows(x.cuda())
    _wgrad_check(p, b, off, janus.packed_wgrad(p, b.cuda(), off.cuda()), "f16")


@pytest.mark.parametrize("t", TYPES)
def test_wgrad_many_rows(t):
    """Long groups (several chunks each) and the same result on every run."""
    import torch
    from paper_2604_15821_amd import janus
    banner("packed_wgrad long", t)
    x, b, off = _wgrad_case(1, [20_000, 5, 9_000], 64, 96, t)
    p = janus.pack_rows(x.cuda())
    b_, off_ = b.cuda(), off.cuda()
    G = janus.packed_wgrad(p, b_, off_)
    _wgrad_check(p, b, off, G, t)
    for _ in range(3):
        assert torch.equal(G, janus.packed_wgrad(p, b_, off_))


@pytest.mark.parametrize("t", TYPES)
def test_wgrad_strides_and_rows_behind_the_last_group(t):
    import torch
    from paper_2604_15821_amd import janus
    for ldb, ldq, shift in ((77, 61, 0), (80, 64, 0), (83, 70, 3)):
        banner("packed_wgrad strides", t, ldb, ldq, shift)
        x, b, off = _wgrad_case(3, [50, 20], 60, 70, t, pad=13)
        b[70:] = float("nan")
        x[70:] = float("nan")
        q = torch.full((83, ldq + shift), -128, dtype=torch.int8, device="cuda:0")
        code = torch.full((83, 4), 255, dtype=torch.uint8, device="cuda:0")
        p = janus.pack_rows(x.cuda(), out=janus.PackedRows(q[:, shift:shift + 60], code[:, :2]))
        wide = torch.full((83, ldb + shift), float("nan"), dtype=_dt(t), device="cuda:0")
        wide[:, shift:shift + 70] = b.cuda()
        G = janus.packed_wgrad(p, wide[:, shift:shift + 70], off.cuda())
        _wgrad_check(p, b, off, G, t)


def test_wgrad_nan_reaches_its_own_row_and_column():
    import torch
    from paper_2604_15821_amd import janus
    banner("packed_wgrad nan")
    x, b, off = _wgrad_case(5, [200, 100], 128, 96, "f32")
    p0 = janus.pack_rows(x.cuda())
    G0 = janus.packed_wgrad(p0, b.cuda(), off.cuda())
    x[10, 40] = float("inf")       # block 32..63 of group 0
    b[250, 7] = float("nan")       # column 7 of group 1
    b[20, 9] = float("inf")        # column 9 of group 0
    G = janus.packed_wgrad(janus.pack_rows(x.cuda()), b.cuda(), off.cuda())
    bad = torch.zeros(2, 128, 96, dtype=torch.bool)
    bad[0, 32:64] = True
    bad[1, :, 7] = True
    bad[0, :, 9] = True
    got, ref = G.cpu(), G0.cpu()
    assert not torch.isfinite(got[bad]).any()
    assert torch.equal(got[~bad], ref[~bad])


def test_wgrad_large_values_and_empty():
    import torch
    from paper_2604_15821_amd import janus
    banner("packed_wgrad range")
    x = torch.full((4, 32), 2.0 ** 60).cuda()
    b = torch.full((4, 16), 2.0 ** -80).cuda()
    off = torch.tensor([0, 0, 4, 4], dtype=torch.int32).cuda()
    G = janus.packed_wgrad(janus.pack_rows(x), b, off)
    assert (G[1] == 2.0 ** -18).all() and (G[0] == 0).all() and (G[2] == 0).all()
    none = torch.zeros(0, 32, device="cuda:0")
    G = janus.packed_wgrad(janus.pack_rows(none), none, torch.zeros(3, dtype=torch.int32, device="cuda:0"))
    assert G.shape == (2, 32, 32) and (G == 0).all()
