"""Operators on rows of tokens, the part that needs no GPU: the format of the checkpoints, what the calls refuse, workspace sizes, and the
formulas of the backward passes against differences."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_1707_04585_b200 import binding as B
from tests import token_ref as ref

INVALID, SHAPE, SMALL, MISALIGNED = -1, -2, -3, -4


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(-1)                # planning only: everything in front of a launch
    yield c
    c.close()


# ------------------------------------------------------------------ the format
@pytest.mark.parametrize("rows,channels", [(0, 1), (1, 1), (1, 32), (1, 33), (64, 128), (65, 129), (1000, 4096), (1 << 20, 4096)])
def test_checkpoint_bytes(ctx, rows, channels):
    n = B.revnet_act_ckpt_bytes(ctx, rows, channels)
    assert n == ref.layout(rows, channels)[4] == B._ck_bytes(rows, channels)
    if rows >= 1000:
        assert n <= 1.04 * rows * channels


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_every_value_held_is_a_bf16_number_and_within_half_a_step(code):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((200, 96)) * np.exp(6 * rng.standard_normal((200, 1)))
    x[0] = 0
    x[1] *= 1e-37
    x = x.astype(np.float32).astype(np.float64)
    c, s = ref.encode(x, code)
    v = ref.decode(c, s, 96, code)
    assert torch.equal(v, v.to(torch.bfloat16).double())
    assert (torch.from_numpy(x) - v).abs().le(ref.half_step(c, s, 96, code)).all()
    # the scale is the smallest that fits: at half of it the largest magnitude would be out of range
    top = np.abs(x.reshape(200, 3, 32)).max(2)
    scale = 2.0 ** (s.astype(float) - 127)
    assert (top <= ref.TOP[code] * scale).all() and ((top > ref.TOP[code] * scale / 2) | (s == 10)).all()


def test_codes_by_hand():
    x = np.zeros((1, 32))
    x[0, :6] = [127, -127, 0.5, 1.5, -0.5, 2.5]                  # ties to even
    c, s = ref.encode(x, "int8")
    assert s[0, 0] == 127 and list(c.view(np.int8)[0, :6]) == [127, -127, 0, 2, 0, 2]
    x[0, 0] = 127.00001
    assert ref.encode(x, "int8")[1][0, 0] == 128
    x[0, :5] = [448, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10]  # halfway between 1 and 1.125; 1.125 and 1.25; 0 and 2^-9; 2^-9 and 2^-8
    c, s = ref.encode(x, "e4m3")
    assert s[0, 0] == 127 and list(ref.code_values(c, "e4m3")[0, :5]) == [448, 1.0, 1.25, 0.0, 2.0 ** -8]
    x[0, 3] = np.inf
    c, s = ref.encode(x, "e4m3")
    assert s[0, 0] == 255 and not c.any()
    assert torch.equal(torch.tensor([1.0625, 448.0, -3 * 2.0 ** -10]).to(torch.float8_e4m3fn).float().double(),
                       torch.from_numpy(ref.code_values(ref._e4m3_code(np.array([1.0625, 448.0, -3 * 2.0 ** -10])), "e4m3")))


# ------------------------------------------------------------------ refusals
FAKE = 0x10000                       # an address that is never followed: every call here is refused first


def call(ctx, name, desc, *ptrs, ws=None):
    args = [C.c_void_p(p) for p in ptrs] + ([C.c_void_p(ws[0]), C.c_size_t(ws[1])] if ws else [])
    return getattr(B.lib(), name)(ctx.h, C.byref(desc) if desc is not None else None, *args, C.c_void_p(0))


BAD_ACT = [(dict(rows=-1), INVALID), (dict(dtype=2), INVALID), (dict(code=2), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID),
           (dict(channels=0), SHAPE), (dict(channels=(1 << 20) + 1), SHAPE), (dict(channels=33, act=4), SHAPE), (dict(rows=1 << 31), SHAPE),
           (dict(ld_x=31), INVALID), (dict(ld_a=31), INVALID), (dict(ld_x=-32), INVALID), (dict(ld_x=1 << 41), INVALID)]


@pytest.mark.parametrize("change,status", BAD_ACT)
def test_act_descriptor(ctx, change, status):
    d = B.act_desc(4, 32)
    for k, v in change.items():
        setattr(d, k, v)
    assert call(ctx, "revnet_act_store", d, FAKE, FAKE, 0) == status
    assert call(ctx, "revnet_act_load", d, FAKE, FAKE) == status
    assert call(ctx, "revnet_act_bwd", d, FAKE, FAKE, FAKE, 0) == status
    assert "descriptor" in B.lib().revnet_last_error(ctx.h).decode()


def test_act_pointers(ctx):
    d = B.act_desc(4, 32, "f32")
    for args in ((0, FAKE, 0), (FAKE, 0, 0)):
        assert call(ctx, "revnet_act_store", d, *args) == INVALID
    for args in ((FAKE + 2, FAKE, 0), (FAKE, FAKE + 128, 0), (FAKE, FAKE, FAKE + 1)):
        assert call(ctx, "revnet_act_store", d, *args) == MISALIGNED
    for args in ((0, FAKE), (FAKE, 0)):
        assert call(ctx, "revnet_act_load", d, *args) == INVALID
    assert call(ctx, "revnet_act_load", d, FAKE + 16, FAKE) == MISALIGNED
    for args in ((0, FAKE, FAKE, 0), (FAKE, 0, FAKE, 0), (FAKE, FAKE, 0, 0), (FAKE, FAKE, FAKE, FAKE)):
        assert call(ctx, "revnet_act_bwd", d, *args) == INVALID
    assert call(ctx, "revnet_act_bwd", d, FAKE, FAKE, FAKE, FAKE + 64) == MISALIGNED
    assert call(ctx, "revnet_act_store", None, FAKE, FAKE, 0) == INVALID
    # a planning-only context has no device
    assert call(ctx, "revnet_act_store", d, FAKE, FAKE, 0) == INVALID
    assert "device" in B.lib().revnet_last_error(ctx.h).decode()
    d.rows = 0                       # nothing to do
    assert call(ctx, "revnet_act_store", d, 0, 0, 0) == 0 and call(ctx, "revnet_act_load", d, 0, 0) == 0 and call(ctx, "revnet_act_bwd", d, 0, 0, 0, 0) == 0


BAD_NORM = [(dict(rows=-1), INVALID), (dict(stream_dtype=7), INVALID), (dict(branch_dtype=-1), INVALID), (dict(stream_dtype=1, branch_dtype=0), INVALID),
            (dict(code=9), INVALID), (dict(ck_scaled=2), INVALID), (dict(eps=0.0), INVALID), (dict(eps=math.inf), INVALID), (dict(eps=math.nan), INVALID),
            (dict(channels=0), SHAPE), (dict(channels=16385), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(ld_stream=3), INVALID), (dict(ld_branch=3), INVALID)]


@pytest.mark.parametrize("change,status", BAD_NORM)
def test_norm_descriptor(ctx, change, status):
    d = B.norm_desc(4, 32)
    for k, v in change.items():
        setattr(d, k, v)
    assert call(ctx, "revnet_rmsnorm_fwd", d, FAKE, FAKE, 0, 0, 0, 0, 0) == status
    assert call(ctx, "revnet_rmsnorm_bwd", d, FAKE, 0, FAKE, 0, 0, 0, FAKE, 0, 0, ws=(FAKE, 1 << 20)) == status
    assert B.lib().revnet_rmsnorm_workspace_bytes(ctx.h, C.byref(d), C.byref(C.c_size_t())) == status


def test_norm_pointers(ctx):
    d = B.norm_desc(4, 32)
    assert call(ctx, "revnet_rmsnorm_fwd", d, 0, FAKE, 0, 0, 0, 0, 0) == INVALID
    assert call(ctx, "revnet_rmsnorm_fwd", d, FAKE, 0, 0, FAKE, 0, 0, 0) == INVALID          # h without r
    assert call(ctx, "revnet_rmsnorm_fwd", d, FAKE + 2, FAKE, 0, 0, 0, 0, 0) == MISALIGNED
    assert call(ctx, "revnet_rmsnorm_fwd", d, FAKE, FAKE, 0, 0, 0, FAKE + 32, 0) == MISALIGNED
    w = (FAKE, 1 << 20)
    # dn, dh, h, ck, rstd, gamma, dx, dr, dgamma
    for args in ((0, 0, FAKE, 0, 0, 0, FAKE, 0, 0), (FAKE, 0, FAKE, 0, 0, 0, 0, 0, 0), (FAKE, 0, 0, FAKE, 0, 0, FAKE, 0, 0), (FAKE, 0, 0, 0, 0, 0, FAKE, 0, 0),
                 (FAKE, 0, FAKE, FAKE, FAKE, 0, FAKE, 0, 0), (FAKE, 0, FAKE, 0, FAKE, 0, FAKE, 0, 0)):
        assert call(ctx, "revnet_rmsnorm_bwd", d, *args, ws=w) == INVALID
    full = (FAKE, 0, FAKE, 0, 0, 0, FAKE, 0, FAKE)
    need = B.revnet_rmsnorm_workspace_bytes(ctx, d)
    assert call(ctx, "revnet_rmsnorm_bwd", d, *full, ws=(0, 0)) == INVALID
    assert call(ctx, "revnet_rmsnorm_bwd", d, *full, ws=(FAKE, need - 1)) == SMALL
    assert call(ctx, "revnet_rmsnorm_bwd", d, *full, ws=(FAKE + 8, need)) == MISALIGNED
    d.ck_scaled = 1                  # the backward pass cannot take gamma out again
    assert call(ctx, "revnet_rmsnorm_bwd", d, FAKE, 0, 0, FAKE, FAKE, 0, FAKE, 0, 0, ws=w) == INVALID


BAD_WGRAD = [(dict(rows=-1), INVALID), (dict(dy_dtype=3), INVALID), (dict(code=-1), INVALID), (dict(cin=0), SHAPE), (dict(cout=0), SHAPE),
             (dict(cin=65537), SHAPE), (dict(cout=65537), SHAPE), (dict(rows=1 << 29), SHAPE), (dict(rows=(1 << 29) - 1, cout=40), SHAPE), (dict(ld_dy=31), INVALID)]


@pytest.mark.parametrize("change,status", BAD_WGRAD)
def test_wgrad_descriptor(ctx, change, status):
    d = B.wgrad_desc(4, 32, 32)
    for k, v in change.items():
        setattr(d, k, v)
    assert call(ctx, "revnet_linear_wgrad", d, FAKE, FAKE, 0, FAKE, ws=(FAKE, 1 << 30)) == status
    assert B.lib().revnet_linear_wgrad_workspace_bytes(ctx.h, C.byref(d), C.byref(C.c_size_t())) == status


def test_wgrad_pointers_and_workspace(ctx):
    d = B.wgrad_desc(100, 40, 24)
    need = B.revnet_linear_wgrad_workspace_bytes(ctx, d)
    for args in ((0, FAKE, 0, FAKE), (FAKE, 0, 0, FAKE), (FAKE, FAKE, 0, 0)):
        assert call(ctx, "revnet_linear_wgrad", d, *args, ws=(FAKE, need)) == INVALID
    assert call(ctx, "revnet_linear_wgrad", d, FAKE, FAKE, 0, FAKE, ws=(FAKE, need - 1)) == SMALL
    assert call(ctx, "revnet_linear_wgrad", d, FAKE, FAKE, 0, FAKE, ws=(0, need)) == INVALID
    for args, ws in (((FAKE + 1, FAKE, 0, FAKE), FAKE), ((FAKE, FAKE + 16, 0, FAKE), FAKE), ((FAKE, FAKE, 0, FAKE + 4), FAKE), ((FAKE, FAKE, 0, FAKE), FAKE + 4)):
        assert call(ctx, "revnet_linear_wgrad", d, *args, ws=(ws, need)) == MISALIGNED
    d.ld_dy = 32                     # bf16 rows that the loads take from where they are
    need = B.revnet_linear_wgrad_workspace_bytes(ctx, d)
    assert call(ctx, "revnet_linear_wgrad", d, FAKE + 8, FAKE, 0, FAKE, ws=(FAKE, need)) == MISALIGNED
    # the parts of the tiles that the SMs share are bounded, whatever the sizes; only other rows are laid out anew
    assert B.revnet_linear_wgrad_workspace_bytes(ctx, B.wgrad_desc(1 << 20, 4096, 4096)) <= 160 << 20
    assert (1 << 20) * 4096 * 2 < B.revnet_linear_wgrad_workspace_bytes(ctx, B.wgrad_desc(1 << 20, 4096, 4096, ld_dy=4097)) <= (1 << 20) * 4096 * 2 + (160 << 20)


BAD_LOGP = [(dict(rows=-1), INVALID), (dict(dtype=2), INVALID), (dict(vocab=0), SHAPE), (dict(vocab=(1 << 24) + 1), SHAPE), (dict(rows=1 << 31), SHAPE),
            (dict(k=33), INVALID), (dict(k=-1), INVALID), (dict(vocab=5, ld=5, k=6), INVALID), (dict(ld=99), INVALID)]


@pytest.mark.parametrize("change,status", BAD_LOGP)
def test_logprob_descriptor(ctx, change, status):
    d = B.logprob_desc(4, 100, "f32", 5)
    for k, v in change.items():
        setattr(d, k, v)
    assert call(ctx, "revnet_logprobs_fwd", d, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE) == status
    assert call(ctx, "revnet_logprobs_bwd", d, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE) == status


def test_logprob_pointers(ctx):
    d = B.logprob_desc(4, 100, "f32", 5)
    for args in ((0, FAKE, FAKE, 0, 0, FAKE, FAKE), (FAKE, 0, FAKE, 0, 0, FAKE, FAKE), (FAKE, FAKE, FAKE, 0, 0, 0, FAKE), (FAKE, FAKE, FAKE, 0, 0, FAKE, 0)):
        assert call(ctx, "revnet_logprobs_fwd", d, *args) == INVALID
    assert call(ctx, "revnet_logprobs_fwd", d, FAKE + 2, FAKE, FAKE, 0, 0, FAKE, FAKE) == MISALIGNED
    for args in ((0, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE), (FAKE, 0, FAKE, FAKE, FAKE, FAKE, FAKE), (FAKE, FAKE, 0, FAKE, FAKE, FAKE, FAKE),
                 (FAKE, FAKE, FAKE, 0, FAKE, FAKE, FAKE), (FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0)):
        assert call(ctx, "revnet_logprobs_bwd", d, *args) == INVALID
    assert call(ctx, "revnet_logprobs_bwd", d, FAKE, FAKE + 1, FAKE, FAKE, FAKE, FAKE, FAKE) == MISALIGNED


def test_kept_input_of_a_stored_layer(ctx):
    d = B.TransitionDesc(2, 6, 6, 16, 24, 3, 2, 1, 1e-5, 0, 16)
    kept, ws = B.revnet_transition_kept_bytes(ctx, d)
    assert kept == 2 * ((B._ck_bytes(72, 8) + 255) // 256 * 256)
    assert ws >= B.revnet_transition_workspace_bytes(ctx, d)[1] + 72 * 16 * 4
    big = B.TransitionDesc(64, 28, 28, 2048, 4096, 3, 2, 1, 1e-5, 0, 16)
    assert B.revnet_transition_kept_bytes(ctx, big)[0] <= 0.27 * 64 * 28 * 28 * 2048 * 4          # of the float32 or fixed-point pair
    lib, P = B.lib(), C.c_void_p

    def keep(*p, code=0):
        return lib.revnet_transition_keep(ctx.h, C.byref(d), P(p[0]), P(p[1]), C.c_int(code), P(p[2]), P(0))

    def bwd(kept_at=FAKE, code=0, size=ws, at=FAKE, **other):
        p = [P(other.get(n, FAKE)) for n in ("dout1", "dout2", "W", "gamma", "beta", "din1", "din2", "dW", "dgamma", "dbeta")]
        return lib.revnet_transition_bwd_kept(ctx.h, C.byref(d), C.c_int(code), P(kept_at), *p, P(at), C.c_size_t(size), P(0))
    assert keep(0, FAKE, FAKE) == INVALID and keep(FAKE, 0, FAKE) == INVALID and keep(FAKE, FAKE, 0) == INVALID and keep(FAKE, FAKE, FAKE, code=2) == INVALID
    assert keep(FAKE + 4, FAKE, FAKE) == MISALIGNED and keep(FAKE, FAKE, FAKE + 16) == MISALIGNED
    assert bwd(kept_at=0) == INVALID and bwd(code=-1) == INVALID and bwd(din2=0) == INVALID and bwd(dW=0) == INVALID
    assert bwd(size=ws - 1) == SMALL and bwd(kept_at=FAKE + 32) == MISALIGNED and bwd(dout1=FAKE + 4) == MISALIGNED
    d.k = 5
    assert keep(FAKE, FAKE, FAKE) == SHAPE and bwd() == SHAPE


def test_binding_checks_tensors_before_their_addresses(ctx):
    """Tensors that do not fit the descriptor never reach the library."""
    x, ck = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(1024, dtype=torch.uint8)
    with pytest.raises(B.RevnetError, match="x must be") as e:
        B.revnet_act_store(ctx, B.act_desc(4, 32), x, ck)                # not on the context's device
    assert e.value.status == INVALID
    with pytest.raises(B.RevnetError, match="logits must be"):
        B.revnet_logprobs_fwd(ctx, B.logprob_desc(4, 32), x, None, None, None, None)
    with pytest.raises(B.RevnetError, match="dy must be"):
        B.revnet_linear_wgrad(ctx, B.wgrad_desc(4, 32, 32), x, ck, None, None, None)
    with pytest.raises(B.RevnetError, match="x must be"):
        B.revnet_rmsnorm_fwd(ctx, B.norm_desc(4, 32), x, None, None, None, None, None, None)


# ------------------------------------------------------------------ formulas against differences
def central(f, x, dy, h=1e-5):
    """Gradient of sum(f(x) dy) by central differences in float64."""
    g = torch.zeros_like(x)
    for i in range(x.numel()):
        for sign in (1, -1):
            y = x.clone()
            y.view(-1)[i] += sign * h
            g.view(-1)[i] += sign * (f(y) * dy).sum() / (2 * h)
    return g


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu", "swiglu"])
def test_activation_gradient(kind):
    torch.manual_seed(1)
    x = torch.randn(3, 10, dtype=torch.float64) * 2
    x = torch.where(x.abs() < 1e-3, x + 0.1, x)      # ReLU's corner has no difference
    da = torch.randn_like(ref.act(x, kind))
    assert torch.allclose(ref.act_bwd(x, da, kind), central(lambda y: ref.act(y, kind), x, da), rtol=1e-7, atol=1e-8)


def test_norm_gradient():
    torch.manual_seed(2)
    h, dn, dh = (torch.randn(3, 9, dtype=torch.float64) for _ in range(3))
    gamma = torch.randn(9, dtype=torch.float64)
    rstd, xh, _ = ref.norm_fwd(h, gamma, 1e-5)
    dx, dgamma = ref.norm_bwd(dn, dh, xh, rstd, gamma)
    assert torch.allclose(dx - dh, central(lambda y: ref.norm_fwd(y, gamma, 1e-5)[2], h, dn), rtol=1e-7, atol=1e-8)
    assert torch.allclose(dgamma, central(lambda g: ref.norm_fwd(h, g, 1e-5)[2], gamma, dn), rtol=1e-7, atol=1e-8)


def test_logprob_gradient():
    torch.manual_seed(3)
    x = torch.randn(4, 7, dtype=torch.float64) * 2
    x[2, 3:5] = -math.inf
    t = torch.tensor([0, 6, 1, -1])
    g, ge = torch.randn(4, dtype=torch.float64), torch.randn(4, dtype=torch.float64)
    lse, _, ent = ref.logprobs(x, t)
    d = ref.logprobs_bwd(x, t, lse, ent, g, ge)
    live = x > -math.inf

    def f(y):
        _, lp, h = ref.logprobs(torch.where(live, y, -math.inf), t)
        return torch.stack([lp, h])
    want = central(f, torch.where(live, x, 0.0), torch.stack([g, ge]))
    assert torch.allclose(d, torch.where(live, want, 0.0), rtol=1e-7, atol=1e-8)
