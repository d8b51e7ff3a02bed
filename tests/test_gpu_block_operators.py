"""The operators around an expert block together, as a training step and a call on a few tokens use
them; captured graphs, streams and calls at once."""
import numpy as np
import pytest

from helpers import banner

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _values(p):
    step = 2.0 ** (p.code.cpu().double() - 127)
    return p.q.cpu().double() * step.repeat_interleave(32, 1)[:, : p.q.shape[1]]


def _unit(v, eps):
    return v / (v * v).mean(1, keepdim=True).add(eps).sqrt()


def test_training_block_from_checkpoints_in_8_bits():
    """Forward through norm, two grouped products with SiLU between and the gated residual norm, then the
    backward pass from packed X, A and S.  Each gradient is compared with its formula in 64 bits at the
    packed values, and the weight gradients with those of the unpacked activations, from which they may
    differ by the packing: at most half a scale step per activation times the gradient's magnitude."""
    import torch
    from paper_2604_15821_amd import janus
    from paper_2604_15821_amd.synth import WORKLOADS
    banner("block training")
    G, d, h, eps = 4, 128, 256, 1e-6
    sizes = [300, 0, 77, 450]
    rows = sum(sizes)
    g = torch.Generator().manual_seed(0)
    R = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    h0, W1, W2 = R(rows, d), R(G, d, h) / d ** 0.5, R(G, h, d) / h ** 0.5
    w_in, w_post, scale, w_next = 1 + 0.1 * R(d), 1 + 0.1 * R(d), 0.3 + 0.1 * R(d), 1 + 0.1 * R(d)
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32))
    seqs = torch.tensor([0, 100, 100, 500, rows], dtype=torch.int32)
    gate, dr, dn = R(4, d), R(rows, d), R(rows, d)
    c = lambda t: t.cuda()  # noqa: E731
    ctx = janus.Context(WORKLOADS["tiny"].model)
    try:
        # the norm before the block is the n of a residual update with nothing added
        _, X = janus.residual_norm(c(h0), torch.zeros(rows, d, device="cuda:0"), w_pre=c(w_in), eps=eps)
        A = ctx.grouped_gemm(X, c(W1), c(off), d, h, 0)
        pX, pA = janus.pack_rows(X), janus.pack_rows(A)
        S = A * torch.sigmoid(A)
        Y = ctx.grouped_gemm(S, c(W2), c(off), h, d, 0)
        p = dict(w_post=c(w_post), gate=c(gate), gate_off=c(seqs), scale=c(scale), w_pre=c(w_next), eps=eps)
        r, n = janus.residual_norm(c(h0), Y, **p)
        back = janus.residual_norm_grad(c(dr), c(dn), r, Y, **p)
        dS = ctx.grouped_gemm(back.db, c(W2), c(off), d, h, 1)
        dA, S8 = janus.unpack_rows(pA, torch.float32, act="silu", grad=dS, value=True)
        pS = janus.pack_rows(S8)
        dW2 = janus.packed_wgrad(pS, back.db, c(off))
        dW1 = janus.packed_wgrad(pX, dA, c(off))
        torch.cuda.synchronize()
    finally:
        ctx.close()
    X_, A_, S_, Y_, db_, dA_, dS_ = [v.cpu().double() for v in (X, A, S, Y, back.db, dA, dS)]
    assert (X_ - _unit(h0.double(), eps) * w_in).abs().max() <= 64 * E * X_.abs().max()
    a8 = _values(pA)
    s8 = torch.sigmoid(a8)
    assert (dA_ - dS_ * (s8 + a8 * s8 * (1 - s8))).abs().max() <= 64 * E * (1 + a8.abs().max()) * dS_.abs().max()
    for grad, held, was, up in ((dW2, pS, S_, db_), (dW1, pX, X_, dA_)):
        v = _values(held)
        for q, (m0, m1) in enumerate(zip(off.tolist(), off.tolist()[1:])):
            got = grad[q].cpu().double()
            want, size = v[m0:m1].t() @ up[m0:m1], v[m0:m1].abs().t() @ up[m0:m1].abs()
            assert ((got - want).abs() <= (6 * (m1 - m0) + 64) * E * size).all()
            true = was[m0:m1].t() @ up[m0:m1]
            if held is pX:   # half a step per value; S8 carries the rounding of A as well
                half = (2.0 ** (held.code.cpu().double() - 128)).repeat_interleave(32, 1)[:, :v.shape[1]]
                assert ((got - true).abs() <= half[m0:m1].t() @ up[m0:m1].abs() + (6 * (m1 - m0) + 64) * E * size).all()


def test_few_tokens_block():
    """One block of inference: residual_norm gives the layer its input, the layer's output goes into the next
    residual_norm; compared with the formulas in 64 bits, the layer at the gates and experts it chose."""
    import torch
    from paper_2604_15821_amd import janus
    banner("block few tokens")
    d, h, n, k, eps = 128, 256, 8, 2, 1e-6
    g = torch.Generator().manual_seed(2)
    R = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    h0, b0 = R(11, d), R(11, d)
    router, W1, W2 = R(d, n) / d ** 0.5, R(n, d, h) / d ** 0.5, R(n, h, d) / h ** 0.5
    w1, w2, w3 = 1 + 0.1 * R(d), 1 + 0.1 * R(d), 0.5 + 0.1 * R(d)
    c = lambda t: t.cuda()  # noqa: E731
    r1, x = janus.residual_norm(c(h0), c(b0), w_pre=c(w1), eps=eps)
    y, eid, gate = janus.expert_layer(x, c(router), c(W1), c(W2), k)
    r2, _ = janus.residual_norm(r1, y, w_post=c(w2), scale=c(w3), eps=eps)
    R1 = h0.double() + b0.double()
    X = _unit(R1, eps) * w1
    rows = []
    for m in range(11):
        a = [X[m] @ W1[q].double() for q in eid[m].tolist()]
        rows.append(sum(gate[m, c_].item() * ((v * torch.sigmoid(v)) @ W2[q].double())
                        for c_, (v, q) in enumerate(zip(a, eid[m].tolist()))))
    want = R1 + w3 * w2 * _unit(torch.stack(rows), eps)
    # sums of up to 256 products with standard normal terms, twice, and two norms: 2^-24 times some hundreds
    assert (r2.cpu().double() - want).abs().max() <= 2000 * E * want.abs().max()


def _all_calls(s):
    from paper_2604_15821_amd import janus
    import torch
    r, n = janus.residual_norm(s["x"], s["b"], w_post=s["w"], gate=s["gate"], gate_off=s["seqs"], scale=s["w"], w_pre=s["w"])
    g = janus.residual_norm_grad(s["x"], n, r, s["b"], w_post=s["w"], gate=s["gate"], gate_off=s["seqs"], scale=s["w"], w_pre=s["w"])
    y, eid, gate = janus.expert_layer(n[:24], s["router"], s["W1"], s["W2"], 2)
    p = janus.pack_rows(n)
    v, t = janus.unpack_rows(p, torch.float32, act="silu", grad=r, value=True)
    G = janus.packed_wgrad(p, g.db, s["off"])
    return [r, n, *g, y, eid, gate, p.q, p.code, v, t, G]


def _state(seed, rows=5000, d=128):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    R = lambda *s: torch.randn(*s, generator=g, device="cuda:0")  # noqa: E731
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")  # noqa: E731
    return dict(x=R(rows, d), b=R(rows, d), w=R(d), gate=R(3, d), seqs=i([0, 7, 4000, rows]), router=R(d, 8) / 11,
                W1=R(8, d, 64) / 11, W2=R(8, 64, d) / 8, off=i([0, 1000, 1000, rows]))


def test_captured_graph_replayed():
    """One graph of every operator, replayed on new inputs with eager work between, is the eager result;
    a second graph of the same calls, replayed beside it on another stream, has its own scratch memory."""
    import torch
    banner("block graph")
    states = [_state(k) for k in range(4)]
    want = [[t.clone() for t in _all_calls(s)] for s in states]
    bufs = [{k: v.clone() for k, v in states[0].items()} for _ in range(2)]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for b in bufs:
            _all_calls(b)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for b in bufs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(_all_calls(b))
        graphs.append(gr)
    for k in (1, 2, 3, 1):
        for b, s in zip(bufs, (states[k], states[(k + 1) % 4])):
            for name, v in s.items():
                b[name].copy_(v)
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for out, ref in zip(outs, (want[k], want[(k + 1) % 4])):
            for a, c in zip(out, ref):
                assert torch.equal(a, c)
        eager = _all_calls(states[k])
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, want[k]))


def test_two_streams_at_once():
    import torch
    banner("block streams")
    states = [_state(k) for k in range(2)]
    want = [[t.clone() for t in _all_calls(s)] for s in states]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k] = _all_calls(states[k])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_rows_beyond_32_bit_offsets():
    """Rows 2^26 values apart, 35 of them: byte and element offsets past 2^31."""
    import torch
    from paper_2604_15821_amd import janus
    banner("block large offsets: norm, pack, unpack")
    rows, d, ld = 35, 72, 1 << 26
    g = torch.Generator(device="cuda:0").manual_seed(3)
    small = torch.randn(rows, d, generator=g, device="cuda:0").bfloat16()
    wide = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda:0")
    x = wide.as_strided((rows, d), (ld, 1))
    x.copy_(small)
    b, w = torch.randn(rows, d, generator=g, device="cuda:0").bfloat16(), torch.rand(d, generator=g, device="cuda:0")
    want = janus.residual_norm(small, b, w_post=w, w_pre=w)
    got = janus.residual_norm(x, b, w_post=w, w_pre=w, out=(x, torch.empty_like(b)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    back = janus.residual_norm_grad(small, b, x, b, w_post=w, w_pre=w)
    ref = janus.residual_norm_grad(small, b, want[0], b, w_post=w, w_pre=w)
    assert all(torch.equal(p, q) for p, q in zip(back, ref) if q is not None)
    q = torch.empty(rows * ld, dtype=torch.int8, device="cuda:0").as_strided((rows, d), (ld, 1))
    code = torch.empty(rows, 3, dtype=torch.uint8, device="cuda:0")
    p = janus.pack_rows(x, out=janus.PackedRows(q, code))
    ref = janus.pack_rows(want[0])
    assert torch.equal(p.q, ref.q) and torch.equal(p.code, ref.code)
    assert torch.equal(janus.unpack_rows(p, torch.bfloat16, act="silu", grad=x, out=x),
                       janus.unpack_rows(ref, torch.bfloat16, act="silu", grad=want[0]))


def test_weight_gradient_beyond_32_bit_offsets():
    import torch
    from paper_2604_15821_amd import janus
    banner("block large offsets: weight gradient")
    rows, P, Q, ld = 60_000, 40, 24, 40_000
    g = torch.Generator(device="cuda:0").manual_seed(4)
    small = torch.randn(rows, Q, generator=g, device="cuda:0").bfloat16()
    B = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda:0").as_strided((rows, Q), (ld, 1))
    B.copy_(small)
    p = janus.pack_rows(torch.randn(rows, P, generator=g, device="cuda:0"))
    off = torch.tensor([0, 1000, rows - 7, rows], dtype=torch.int32, device="cuda:0")
    out = torch.full((3, P, Q), float("nan"), device="cuda:0")
    assert janus.packed_wgrad(p, B, off, out=out) is out
    assert torch.equal(out, janus.packed_wgrad(p, small, off))


def test_expert_weights_beyond_32_bit_offsets():
    """The last of 17 experts begins past 2^31 values; only its weights are filled."""
    import torch
    from paper_2604_15821_amd import janus
    banner("block large offsets: expert layer")
    n, d, h, tokens = 17, 2048, 65_536, 3
    g = torch.Generator(device="cuda:0").manual_seed(5)
    up = torch.empty(n, d, h, dtype=torch.bfloat16, device="cuda:0")
    down = torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda:0")
    up[16] = torch.randn(d, h, generator=g, device="cuda:0") / d ** 0.5
    down[16] = torch.randn(h, d, generator=g, device="cuda:0") / h ** 0.5
    x = torch.randn(tokens, d, generator=g, device="cuda:0").bfloat16()
    beta = torch.full((n,), -float("inf"), device="cuda:0")
    beta[16] = 0.0
    y, eid, gate = janus.expert_layer(x, torch.zeros(d, n, device="cuda:0"), up, down, 1, beta=beta)
    assert (eid == 16).all() and (gate == 1).all()
    a = x.float() @ up[16].float()
    s = a * torch.sigmoid(a)
    want = s.double().cpu() @ down[16].cpu().double()
    size = s.abs().double().cpu() @ down[16].cpu().double().abs()
    # fp32 pre-activations on both sides (2 (d + 8) e of their magnitudes, of the order of sqrt(d) times the value), the
    # hidden values to 2^-16, the sum of h products, and the rounding to bf16
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -16 + 2 * (h + 8) * E + 4 * (d + 8) * E) * size
    assert ((y.cpu().double() - want).abs() <= tol).all()
