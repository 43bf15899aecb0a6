"""Refusals of the operators on rows of tokens where there are no rows: parameters' gradients are written all the same."""
import pytest

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
