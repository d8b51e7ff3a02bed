"""Sizes that the operators around an expert block cannot count in 32 bits are refused, by the library and by the
binding, whose arguments the library would see cut off (CPU)."""
import pytest
import torch

from paper_2604_15821_amd import janus

EUNSUP = janus.JANUS_EUNSUPPORTED
P = 1 << 20   # an address that no refused call reads
WIDEST = 2 ** 31 - 4097


@pytest.mark.parametrize("d", [WIDEST + 1, 2 ** 31 - 2049, 2 ** 31 - 31, 2 ** 31 - 1])
def test_packed_widths(d):
    lib = janus._lib()
    assert lib.janus_pack_rows(P, d, 0, 1, d, P, d, P, d // 32 + 1, None) == EUNSUP
    assert lib.janus_unpack_rows(P, d, P, d // 32 + 1, 1, d, 0, 0, None, 0, None, 0, P, d, None) == EUNSUP
    assert lib.janus_packed_wgrad(P, d, P, d // 32 + 1, P, 1, 0, P, P, 1, 1, d, 1, P, 1 << 62, None) == EUNSUP
    # the widest rows pass to the next check
    assert lib.janus_pack_rows(P, WIDEST - 1, 0, 1, WIDEST, P, WIDEST, P, WIDEST // 32 + 1, None) == janus.JANUS_EINVAL


def _meta(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_binding_counts():
    wide = 2 ** 32 + 16
    x = _meta(1, wide)
    p = janus.PackedRows(_meta(1, wide, dtype=torch.int8), _meta(1, (wide + 31) // 32, dtype=torch.uint8))
    for call in (lambda: janus.pack_rows(x), lambda: janus.unpack_rows(p, torch.float32), lambda: janus.residual_norm(x, x),
                 lambda: janus.residual_norm_grad(x, None, None, x),
                 lambda: janus.packed_wgrad(p, x, _meta(2, dtype=torch.int32)),
                 lambda: janus.expert_layer(x, _meta(wide, 1), _meta(1, wide, 16), _meta(1, 16, wide), 1)):
        with pytest.raises(ValueError, match="columns"):
            call()
    y = _meta(1, 16)
    for n, h, k, word in ((wide, 16, 1, "w_up"), (1, wide, 1, "w_up"), (1, 16, wide + 1, "top_k"), (1, 16, -wide + 1, "top_k"),
                          (1, 16, 2 ** 31, "top_k")):
        with pytest.raises(ValueError, match=word):
            janus.expert_layer(y, _meta(16, n), _meta(n, 16, h), _meta(n, h, 16), k)
    for name in ("row_off", "gate_off"):
        with pytest.raises(ValueError, match=f"{name}: .* at most"):
            janus._offsets(_meta(wide, dtype=torch.int32), name, y.device)


@pytest.mark.parametrize("rows", [1, 10_000, 1 << 24, 2 ** 31 - 4097])
def test_distances_of_rows_up_to_256_kib(rows):
    """The packed weight gradient takes rows 262 144 bytes apart at any number of rows (the call then asks for its
    scratch memory, which is not given), and no more than its 32-bit offsets reach at the longest chunks."""
    lib = janus._lib()

    def call(ldq, ldc, ldb, t):
        return lib.janus_packed_wgrad(P, ldq, P, ldc, P, ldb, t, P, P, 1, rows, 40, 24, None, 0, None)
    far = 1 << 18
    for t, size in ((0, 4), (1, 2), (2, 2)):
        for ld in ((far, 2, 24), (40, far, 24), (40, 2, far // size), (far, far, far // size)):
            assert call(*ld, t) == janus.JANUS_EINVAL, ld
        for ld in ((1 << 23, 2, 24), (40, 1 << 23, 24), (40, 2, (1 << 23) // size), (40, 2, (1 << 62) + 24)):
            assert call(*ld, t) == EUNSUP, ld
        if rows >= 1 << 24:
            assert call(263_000, 2, 24, t) == EUNSUP
