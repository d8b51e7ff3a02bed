"""Refusals of the operators around an expert block: the library's return codes for arguments that it
can judge on the host, and the binding's checks before an address reaches the library (CPU)."""
import ctypes as C

import pytest
import torch

from paper_2604_15821_amd import janus

EINVAL, EUNSUP = janus.JANUS_EINVAL, janus.JANUS_EUNSUPPORTED
P = 1 << 20   # an address that no refused call reads


def _norm(**over):
    p = janus.Norm(4, 64, 0, 1e-6, 0, P, P, P, None, 64, None)
    for k, v in over.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), EINVAL), (dict(rows=1 << 31), EINVAL), (dict(d=0), EINVAL), (dict(d=8193), EUNSUP),
    (dict(type=3), EINVAL), (dict(type=-1), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(gate_off=P), EINVAL), (dict(gate=P, ldg=63), EINVAL),
    (dict(gate=P, gate_off=P, n_seq=-1), EINVAL)])
def test_norm_settings(over, code):
    lib, p = janus._lib(), _norm(**over)
    assert lib.janus_residual_norm(C.byref(p), P, 64, P, 64, P, 64, P, 64, None) == code
    assert lib.janus_residual_norm_grad_workspace(C.byref(p)) == code
    assert lib.janus_residual_norm_grad(C.byref(p), P, 64, P, 64, P, 64, P, 64, P, 64, P, 64, None, None, None, None, 64,
                                        P, 1 << 40, None) == code


def test_norm_arrays():
    lib, p = janus._lib(), _norm()
    good = [P, 64, P, 64, P, 64, P, 64]
    for k, v in ((0, None), (2, None), (4, None), (6, None), (1, 63), (3, 63), (5, 63), (7, 63)):
        bad = list(good)
        bad[k] = v
        assert lib.janus_residual_norm(C.byref(p), *bad, None) == EINVAL, k
    q = _norm(w_pre=None)
    assert lib.janus_residual_norm(C.byref(q), *good, None) == EINVAL   # n without w_pre
    assert lib.janus_residual_norm(None, *good, None) == EINVAL
    size = lib.janus_residual_norm_grad_workspace(C.byref(p))
    assert size > 0
    grads = [P, 64, P, 64, P, 64, P, 64, P, 64, P, 64, P, P, P, None, 64, P, size]
    #           dn       r        b        dx        db      ld of each            work  size
    for k, v in ((2, None), (4, None), (6, None), (8, None), (10, None), (1, 63), (3, 63), (5, 63), (7, 63), (9, 63),
                 (11, 63), (17, None), (17, P + 8), (18, size - 1), (15, P)):
        bad = list(grads)
        bad[k] = v
        assert lib.janus_residual_norm_grad(C.byref(p), *bad, None) == EINVAL, k
    for name, k in (("w_post", 12), ("scale", 13), ("w_pre", 14)):   # a gradient of what is not there
        q = _norm(**{name: None})
        bad = list(grads)
        if name == "w_pre":
            bad[2] = bad[4] = None
        assert lib.janus_residual_norm_grad(C.byref(q), *bad, None) == EINVAL, name


def _experts(**over):
    p = janus.Experts(64, 128, 8, 2, 0, 0, P, None, P, P)
    for k, v in over.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("over,tokens,code", [
    (dict(d=0), 1, EINVAL), (dict(d_hidden=-16), 1, EINVAL), (dict(n_experts=0), 1, EINVAL), (dict(top_k=0), 1, EINVAL),
    (dict(top_k=9, n_experts=8), 1, EINVAL), (dict(type=7), 1, EINVAL), (dict(normalize=2), 1, EINVAL), ({}, -1, EINVAL),
    (dict(d=72), 1, EUNSUP), (dict(d_hidden=120), 1, EUNSUP), (dict(n_experts=257), 1, EUNSUP),
    (dict(top_k=9, n_experts=16), 1, EUNSUP), ({}, 65, EUNSUP), (dict(d=16400), 1, EUNSUP), (dict(d_hidden=65552), 1, EUNSUP)])
def test_expert_settings(over, tokens, code):
    lib, p = janus._lib(), _experts(**over)
    assert lib.janus_expert_layer_workspace(C.byref(p), tokens) == code
    assert lib.janus_expert_layer(C.byref(p), P, 64, tokens, P, 64, P, P, P, 1 << 40, None) == code


def test_expert_arrays():
    lib, p = janus._lib(), _experts()
    size = lib.janus_expert_layer_workspace(C.byref(p), 3)
    good = [P, 64, 3, P, 64, P, P, P, size]
    for k, v in ((0, None), (3, None), (5, None), (6, None), (7, None), (1, 63), (4, 63), (8, size - 1), (0, P + 4), (3, P + 4),
                 (1, 65), (4, 65), (7, P + 4)):
        bad = list(good)
        bad[k] = v
        assert lib.janus_expert_layer(C.byref(p), *bad, None) == EINVAL, (k, v)
    for name, v in (("router", None), ("w_up", None), ("w_down", None), ("w_up", P + 4), ("w_down", P + 8)):
        assert lib.janus_expert_layer(C.byref(_experts(**{name: v})), *good, None) == EINVAL, name
    assert lib.janus_expert_layer(None, *good, None) == EINVAL


def test_packed_arrays():
    lib = janus._lib()
    good = [P, 40, 0, 4, 40, P, 48, P, 2]
    for k, v in ((0, None), (1, 39), (2, 3), (3, -1), (3, 1 << 31), (4, 0), (5, None), (6, 39), (7, None), (8, 1)):
        bad = list(good)
        bad[k] = v
        assert lib.janus_pack_rows(*bad, None) == EINVAL, (k, v)
    good = [P, 48, P, 2, 4, 40, 0, 1, P, 40, P, 40, P, 40]
    for k, v in ((0, None), (1, 39), (2, None), (3, 1), (4, -1), (5, 0), (6, 9), (7, 2), (7, 0), (8, None), (9, 39), (10, None),
                 (11, 39), (13, 39)):
        bad = list(good)
        bad[k] = v
        assert lib.janus_unpack_rows(*bad, None) == EINVAL, (k, v)
    assert lib.janus_unpack_rows(P, 48, P, 2, 4, 40, 0, 1, None, 0, None, 0, None, 0, None) == EINVAL   # nothing to write
    assert lib.janus_pack_rows(None, 40, 0, 0, 40, None, 48, None, 2, None) == 0                        # no rows
    assert lib.janus_unpack_rows(None, 48, None, 2, 0, 40, 0, 0, None, 0, None, 0, None, 0, None) == 0


def test_packed_wgrad_arrays():
    lib = janus._lib()
    size = lib.janus_packed_wgrad_workspace(4, 2, 40, 24, 0)
    assert size > 0
    good = [P, 48, P, 2, P, 24, 0, P, P, 2, 4, 40, 24, P, size]
    for k, v in ((0, None), (1, 39), (2, None), (3, 1), (4, None), (5, 23), (6, 4), (7, None), (8, None), (9, 0), (9, 1025), (10, -1),
                 (10, 1 << 31), (11, 0), (12, 0), (13, None), (13, P + 4), (14, size - 1)):
        bad = list(good)
        bad[k] = v
        assert lib.janus_packed_wgrad(*bad, None) == EINVAL, (k, v)
    for k in (1, 5):   # rows too far apart for the 32-bit offsets of a chunk
        bad = list(good)
        bad[k] = 1 << 30
        assert lib.janus_packed_wgrad(*bad, None) == EUNSUP, k
    for bad in ((-1, 2, 40, 24, 0), (4, 0, 40, 24, 0), (4, 1025, 40, 24, 0), (4, 2, 0, 24, 0), (4, 2, 40, 0, 0), (4, 2, 40, 24, 3)):
        assert lib.janus_packed_wgrad_workspace(*bad) == EINVAL


def test_packed_wgrad_sizes_beyond_a_launch():
    lib = janus._lib()
    most = 1 << 21   # 2^14 tiles of 128 rows x 1024 groups: 2^24 workgroups, 2^32 threads
    for p_, q_ in ((most, 1), (1, 2 * most), ((1 << 31) - 1, (1 << 31) - 1)):
        assert lib.janus_packed_wgrad_workspace(10, 1024, p_, q_, 1) == EUNSUP, (p_, q_)
        bad = [P, p_, P, p_ // 32 + 1, P, q_, 1, P, P, 1024, 10, p_, q_, P, 1 << 62]
        assert lib.janus_packed_wgrad(*bad, None) == EUNSUP, (p_, q_)
    assert lib.janus_packed_wgrad_workspace(10, 1000, most, 1, 1) > 0


def test_binding_refuses_before_the_library():
    x = torch.zeros(4, 64)
    for call in (lambda: janus.residual_norm(x, x), lambda: janus.residual_norm_grad(x, None, None, x),
                 lambda: janus.pack_rows(x), lambda: janus.expert_layer(x, torch.zeros(64, 2), torch.zeros(2, 64, 64),
                                                                        torch.zeros(2, 64, 64), 1),
                 lambda: janus.packed_wgrad(janus.PackedRows(x.to(torch.int8), torch.zeros(4, 2, dtype=torch.uint8)), x,
                                            torch.zeros(2, dtype=torch.int32)),
                 lambda: janus.unpack_rows(janus.PackedRows(x.to(torch.int8), torch.zeros(4, 2, dtype=torch.uint8)), torch.float32)):
        with pytest.raises(ValueError, match="device"):
            call()
    cpu = x.device
    with pytest.raises(TypeError):
        janus._rows(x.double(), "x", torch.float32, (4, 64), cpu)
    with pytest.raises(ValueError, match="shape"):
        janus._rows(x, "x", torch.float32, (4, 65), cpu)
    with pytest.raises(ValueError, match="shape"):
        janus._rows(x[0], "x", torch.float32, (4, 64), cpu)
    with pytest.raises(TypeError):
        janus._type_of(torch.int32, "x")
    with pytest.raises(TypeError):
        janus._matrix([1.0], "x")
    with pytest.raises(ValueError, match="two dimensions"):
        janus._matrix(x[0], "x")
