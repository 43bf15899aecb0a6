"""Refusals of the operators on rows of tokens: without rows (parameters' gradients are written all the same), and of a layer's kept input."""
import ctypes as C

import pytest
import torch

from paper_1707_04585_b200 import binding as B
from tests.test_token_rows_host import FAKE, INVALID, MISALIGNED, SMALL, call


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(-1)
    yield c
    c.close()


def test_norm_gradient_of_no_rows(ctx):
    d = B.norm_desc(0, 32)
    need = B.revnet_rmsnorm_workspace_bytes(ctx, d)
    nothing = (0,) * 8                               # dn, dh, h, ck, rstd, gamma, dx, dr
    assert call(ctx, "revnet_rmsnorm_bwd", d, *nothing, FAKE + 2, ws=(FAKE, need)) == MISALIGNED      # dgamma is set to zero: an address for floats
    assert call(ctx, "revnet_rmsnorm_bwd", d, *nothing, FAKE, ws=(FAKE + 4, need)) == MISALIGNED
    assert call(ctx, "revnet_rmsnorm_bwd", d, *nothing, FAKE, ws=(FAKE, need - 1)) == SMALL
    assert call(ctx, "revnet_rmsnorm_bwd", d, *nothing, FAKE, ws=(FAKE, need)) == INVALID             # (as far as the device: this context has none)
    assert "device" in B.lib().revnet_last_error(ctx.h).decode()
    w = B.wgrad_desc(0, 40, 24)
    assert call(ctx, "revnet_linear_wgrad", w, 0, 0, 0, FAKE + 4, ws=(0, 0)) == MISALIGNED
    assert call(ctx, "revnet_linear_wgrad", w, 0, 0, 0, 0, ws=(0, 0)) == INVALID


def test_kept_input_of_a_stored_layer_stays_on_its_device(ctx):
    """The calls that keep a layer's input launch on the context's device alone, and take no buffer from elsewhere."""
    d = B.TransitionDesc(2, 6, 6, 16, 24, 3, 2, 1, 1e-5, 0, 16)
    kept, ws = B.revnet_transition_kept_bytes(ctx, d)
    P = C.c_void_p
    lib = B.lib()
    assert lib.revnet_transition_keep(ctx.h, C.byref(d), P(FAKE), P(FAKE), C.c_int(0), P(FAKE), P(0)) == INVALID          # this context has no device
    assert "device" in lib.revnet_last_error(ctx.h).decode()
    assert lib.revnet_transition_bwd_kept(ctx.h, C.byref(d), C.c_int(0), P(FAKE), *[P(FAKE)] * 10, P(FAKE), C.c_size_t(ws), P(0)) == INVALID
    assert "device" in lib.revnet_last_error(ctx.h).decode()
    x = torch.zeros(72, 8)
    for bad in (torch.zeros(kept, dtype=torch.uint8), None):     # in host memory; none at all
        with pytest.raises(B.RevnetError, match="kept") as e:
            B.revnet_transition_keep(ctx, d, x, x, "int8", bad)
        assert e.value.status == INVALID
        with pytest.raises(B.RevnetError, match="kept"):
            B.revnet_transition_bwd_kept(ctx, d, "int8", bad, *[x] * 10, bad)
