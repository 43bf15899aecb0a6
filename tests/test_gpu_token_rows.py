"""Operators on rows of tokens on the GPU against float64 (tests/token_ref.py).  Each tolerance is a bound on float32's rounding errors of the
sums and functions in question, stated beside it; outputs in bf16 may be off by half a step more."""
import math

import pytest
import torch

from paper_1707_04585_b200 import binding as B
from tests import token_ref as ref
from tests.token_ref import DT, HALF, U

pytestmark = pytest.mark.gpu
GUARD = 77.0                         # what lies between and behind the rows before a call, and has to lie there after it


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    B.revnet_check_device(c)
    c.close()


class Rows:
    """A [rows][channels] view into a larger buffer: `pad` elements between rows, `skip` in front of the first, some behind the last."""

    def __init__(self, rows, channels, dtype, pad=0, skip=0, value=None):
        self.ld = channels + pad
        self.buf = torch.full((skip + rows * self.ld + 5,), GUARD, dtype=DT[dtype], device="cuda")
        self.t = self.buf[skip:skip + rows * self.ld].view(rows, self.ld)[:, :channels]
        if value is not None:
            self.t.copy_(value)
        self.out = torch.ones_like(self.buf, dtype=torch.bool)
        self.out[skip:skip + rows * self.ld].view(rows, self.ld)[:, :channels] = False

    def cpu(self):
        return self.t.cpu().double()

    def untouched(self):
        return bool((self.buf[self.out] == GUARD).all())


class Ck:
    """A checkpoint buffer with a guard behind it."""

    def __init__(self, rows, channels, data=None):
        self.rows, self.channels, self.n = rows, channels, ref.layout(rows, channels)[4]
        self.buf = torch.full((self.n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        if data is not None:
            self.buf[:self.n] = data.cuda()
        self.t = self.buf[:self.n]

    def parts(self):
        assert (self.buf[self.n:] == 0xA5).all()
        pitch, at, groups, padded, size = ref.layout(self.rows, self.channels)
        rest = self.t[at:].view(groups, padded, 4)
        assert (rest[:, self.rows:] == 0xA5).all()               # scales of rows behind the last one
        return ref.take_apart(self.t, self.rows, self.channels)

    @classmethod
    def of(cls, x, code, fill=0xA5):
        """From values; unwritten scale bytes hold `fill`, so that a kernel that looks at them shows it."""
        c, s = ref.encode(x.cpu().numpy(), code)
        return cls(*x.shape, ref.put_together(c, s, *x.shape, fill=fill))


def data(rows, channels, dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, channels, generator=g, dtype=torch.float64) * scale * torch.exp(0.5 * torch.randn(channels, generator=g, dtype=torch.float64))
    return x.to(DT[dtype])


def within(got, want, tol, dtype="f32"):
    """|got - want| <= tol + half a step of the output type; infinities and NaN in the same places."""
    want = want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~fine].nan_to_num(), want[~fine].nan_to_num())
    err = (got - want).abs()[fine]
    lim = (tol + (want.abs() + tol) * HALF[dtype] + 2.0 ** -134).expand_as(want)[fine]      # (subnormals have a step of 2^-133 in bf16)
    assert (err <= lim).all(), f"error {err.max():.3e}, worst ratio {(err / lim).max():.3f}"


SHAPES = [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 16, 0, 0), (5, 17, 0, 0), (7, 31, 1, 1), (2, 32, 0, 0), (64, 33, 7, 0), (65, 128, 8, 0), (33, 130, 0, 3), (9, 520, 24, 0),
          (300, 1000, 0, 0), (17, 4104, 8, 8)]


# ------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,channels,pad,skip", SHAPES)
def test_store_writes_the_format_byte_for_byte(ctx, rows, channels, pad, skip, dtype, code):
    x = data(rows, channels, dtype, 1)
    if rows > 2:
        x[0] = 0
        x[1] *= 2.0 ** -120           # scales at their lower limit
        x[2, channels // 2] = 3e38    # and far up
    r, ck = Rows(rows, channels, dtype, pad, skip, x), Ck(rows, channels)
    B.revnet_act_store(ctx, B.act_desc(rows, channels, dtype, code, ld_x=r.ld), r.t, ck.t)
    c, s = ck.parts()
    wc, ws = ref.encode(x.double().numpy(), code)
    assert (s == ws).all()
    assert (ref.code_values(c, code) == ref.code_values(wc, code)).all()          # (-0 and 0 are one value)
    for out in ("f32", "bf16"):
        y = Rows(rows, channels, out, pad, skip)
        B.revnet_act_load(ctx, B.act_desc(rows, channels, out, code, ld_a=y.ld), ck.t, y.t)
        assert torch.equal(y.cpu(), ref.decode(wc, ws, channels, code)) and y.untouched()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_ties_limits_and_non_finite_blocks(ctx, code):
    x = torch.zeros(4, 96)
    x[0, :8] = torch.tensor([127, 0.5, 1.5, 2.5, -0.5, -126.5, 63.5, -127.0])
    x[0, 32:40] = torch.tensor([448, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, -240.0, 464.0, 17.0])
    x[1, 5], x[1, 40], x[2, 95] = math.inf, math.nan, -math.inf
    x[1, 70] = 1.0
    x[3] = torch.finfo(torch.float32).max
    ck, y = Ck(4, 96), Rows(4, 96, "f32")
    B.revnet_act_store(ctx, B.act_desc(4, 96, "f32", code), x.cuda(), ck.t)
    c, s = ck.parts()
    wc, ws = ref.encode(x.double().numpy(), code)
    assert (s == ws).all() and (ref.code_values(c, code) == ref.code_values(wc, code)).all()
    B.revnet_act_load(ctx, B.act_desc(4, 96, "f32", code), ck.t, y.t)
    bad = torch.isnan(y.cpu())
    assert bad[1, :64].all() and not bad[1, 64:].any() and bad[2, 64:].all() and not bad[2, :64].any() and not bad[[0, 3]].any()


# ------------------------------------------------------------------ activations
KINDS = ["none", "relu", "gelu", "silu", "swiglu"]


@pytest.mark.parametrize("code,dtype", [("int8", "f32"), ("e4m3", "bf16")])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,channels,pad,skip", [(1, 2, 0, 0), (5, 34, 0, 0), (7, 96, 1, 1), (3, 64, 0, 0), (65, 160, 8, 0), (33, 1040, 0, 0), (9, 4096, 0, 0), (200, 250, 3, 0)])
def test_activation_forward_and_backward(ctx, rows, channels, pad, skip, kind, code, dtype):
    out = channels // 2 if kind == "swiglu" else channels
    x = data(rows, channels, dtype, 2, 2.0)
    da = data(rows, out, dtype, 3)
    rx, ra, ck = Rows(rows, channels, dtype, pad, skip, x), Rows(rows, out, dtype, pad, skip), Ck(rows, channels)
    d = B.act_desc(rows, channels, dtype, code, kind, ld_x=rx.ld, ld_a=ra.ld)
    B.revnet_act_store(ctx, d, rx.t, ck.t, ra.t)
    c, s = ck.parts()
    wc, ws = ref.encode(x.double().numpy(), code)
    assert (s == ws).all() and (ref.code_values(c, code) == ref.code_values(wc, code)).all()

    def tols(v):
        if kind != "swiglu":
            return ref.act_tol(v, kind)
        g, u = v.chunk(2, 1)
        ta, td = ref.act_tol(g, "silu")
        return ta * u.abs() + U * ref.act(v, kind).abs(), torch.cat([td * u.abs(), ta], 1)
    within(ra.cpu(), ref.act(x.double(), kind), tols(x.double())[0], dtype)
    assert ra.untouched() and rx.untouched()
    # what is kept
    x8 = ref.decode(wc, ws, channels, code)
    B.revnet_act_load(ctx, d, ck.t, ra.t)
    ta, td = tols(x8)
    within(ra.cpu(), ref.act(x8, kind), ta, dtype)
    # backward
    rda, rdx, ack = Rows(rows, out, dtype, pad, skip, da), Rows(rows, channels, dtype, pad, skip), Ck(rows, out)
    B.revnet_act_bwd(ctx, d, ck.t, rda.t, rdx.t, ack.t)
    g = da.double().repeat(1, 2) if kind == "swiglu" else da.double()
    want = ref.act_bwd(x8, da.double(), kind)
    within(rdx.cpu(), want, td * g.abs() + 4 * U * want.abs(), dtype)
    assert rdx.untouched() and rda.untouched()
    a = ref.act(x8, kind)
    cc, cs = ack.parts()
    assert ((ref.decode(cc, cs, out, code) - a).abs() <= ref.half_step(cc, cs, out, code) + 2 * ta + 2.0 ** -130).all()
    top = torch.nn.functional.pad(a.abs(), (0, -out % 32)).view(rows, -1, 32).amax(2)
    tt = torch.nn.functional.pad(2 * ta, (0, -out % 32)).view(rows, -1, 32).amax(2) + 2.0 ** -130
    scale = torch.from_numpy(2.0 ** (cs.astype(float) - 127))
    assert (top <= ref.TOP[code] * scale + tt).all() and ((top >= ref.TOP[code] * scale / 2 - tt) | (torch.from_numpy(cs.astype(int)) == 10)).all()
    # without the second checkpoint, and (ungated) in place
    again = Rows(rows, channels, dtype, pad, skip)
    B.revnet_act_bwd(ctx, d, ck.t, rda.t, again.t)
    assert torch.equal(again.t, rdx.t)
    if kind != "swiglu":
        B.revnet_act_bwd(ctx, d, ck.t, rda.t, rda.t)
        assert torch.equal(rda.t, rdx.t)
        keep = ra.t.clone()
        B.revnet_act_store(ctx, d, rx.t, ck.t, ra.t)
        keep = ra.t.clone()
        B.revnet_act_store(ctx, d, rx.t, ck.t, rx.t)
        assert torch.equal(rx.t, keep)


@pytest.mark.parametrize("skip", range(8))
@pytest.mark.parametrize("channels,pad", [(16, 1), (45, 0), (528, 2), (1043, 0), (1056, 5)])
def test_every_alignment_of_a_row(ctx, channels, pad, skip):
    """Rows that start at every element of 16 bytes, and go on at others: nothing beside them is written, and values land where they belong."""
    test_activation_forward_and_backward(ctx, 11, channels, pad, skip, "silu", "int8", "bf16")
    test_activation_forward_and_backward(ctx, 11, channels, pad, skip, "relu", "e4m3", "f32")
    test_norm_forward(ctx, 11, channels, pad, skip, "f32", "bf16", "int8")
    test_norm_backward(ctx, 11, channels, pad, skip, "bf16", "bf16", "h")
    test_norm_backward(ctx, 11, channels, pad, skip, "f32", "f32", "e4m3")


@pytest.mark.parametrize("code,dtype", [("int8", "f32"), ("e4m3", "bf16")])
@pytest.mark.parametrize("half", [1, 4, 15, 16, 17, 20, 31, 33, 40, 520, 523, 2060])
def test_gated_halves_of_any_length(ctx, half, code, dtype):
    """The second half starts inside a block, inside 16 codes, and on neither's boundary."""
    test_activation_forward_and_backward(ctx, 13, 2 * half, 0, 0, "swiglu", code, dtype)
    test_activation_forward_and_backward(ctx, 13, 2 * half, 3, 1, "swiglu", code, dtype)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_a_bad_block_across_the_gate_stays_in_its_block(ctx, code):
    half = 41                         # blocks of 32: the second one holds the end of g and the start of u
    x = torch.ones(2, 2 * half)
    x[0, 50] = math.nan
    ck, a, da, dx, ack = Ck(2, 2 * half), Rows(2, half, "f32"), torch.ones(2, half).cuda(), Rows(2, 2 * half, "f32"), Ck(2, half)
    d = B.act_desc(2, 2 * half, "f32", code, "swiglu")
    B.revnet_act_store(ctx, d, x.cuda(), ck.t)
    B.revnet_act_load(ctx, d, ck.t, a.t)
    B.revnet_act_bwd(ctx, d, ck.t, da, dx.t, ack.t)
    bad = torch.zeros(2 * half, dtype=torch.bool)
    bad[32:64] = True                 # of g: 32 to 40; of u: 0 to 22
    gone = bad[:half] | bad[half:]
    assert torch.equal(torch.isnan(a.cpu())[0], gone) and not torch.isnan(a.cpu()[1]).any()
    g = torch.isnan(dx.cpu())
    assert torch.equal(g[0, :half], gone) and torch.equal(g[0, half:], bad[:half]) and not g[1].any()
    assert torch.isfinite(ref.held(ack.t, 2, half, code)[1]).all()


def test_relu_stops_infinite_gradients_and_nan_reads_back_as_nan(ctx):
    x, da = torch.full((1, 64), -1.0).cuda(), torch.full((1, 64), math.inf).cuda()
    x[0, 40] = math.nan
    ck, dx = Ck(1, 64), torch.empty(1, 64, device="cuda")
    d = B.act_desc(1, 64, "f32", act="relu")
    B.revnet_act_store(ctx, d, x, ck.t)
    B.revnet_act_bwd(ctx, d, ck.t, da, dx)
    assert (dx[0, :32] == 0).all() and torch.isnan(dx[0, 32:]).all()


# ------------------------------------------------------------------ norm
PAIRS = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")]
NORM_SHAPES = [(1, 1, 0, 0), (1, 4096, 0, 0), (2, 7, 0, 0), (5, 33, 1, 1), (300, 16, 0, 0), (65, 64, 8, 0), (129, 520, 0, 0), (40, 1001, 3, 0), (3, 5000, 0, 0), (2, 16384, 0, 0), (700, 256, 0, 0)]
# relative error of a float32 sum of the squares of a row: 32 products one after another, a tree over 512 threads, the division, the root
ROW = 64 * U


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("stream,branch", PAIRS)
@pytest.mark.parametrize("rows,channels,pad,skip", NORM_SHAPES)
def test_norm_forward(ctx, rows, channels, pad, skip, stream, branch, code):
    x, r = data(rows, channels, stream, 4), data(rows, channels, branch, 5)
    gamma = (1 + 0.2 * torch.randn(channels, generator=torch.Generator().manual_seed(6))).float()
    if rows > 2:
        x[1], r[1] = 0, 0             # a row of zeros: rstd = 1 / sqrt(eps)
    eps = 1e-5
    h = (x.float() + r.float()).to(DT[stream])
    rstd, xh, n = ref.norm_fwd(h.double(), gamma.double(), eps)
    rx, rr = Rows(rows, channels, stream, pad, skip, x), Rows(rows, channels, branch, pad, skip, r)
    oh, on, ors = Rows(rows, channels, stream, pad, skip), Rows(rows, channels, branch, pad, skip), torch.empty(rows, device="cuda")
    for scaled in (False, True):
        ck = Ck(rows, channels)
        d = B.norm_desc(rows, channels, stream, branch, eps, code, scaled, rx.ld, rr.ld)
        B.revnet_rmsnorm_fwd(ctx, d, rx.t, rr.t, gamma.cuda(), oh.t, on.t, ck.t, ors)
        assert torch.equal(oh.t.cpu(), h) and oh.untouched() and on.untouched() and rx.untouched()
        within(ors.cpu().double(), rstd, ROW * rstd)
        within(on.cpu(), n, (ROW + 3 * U) * n.abs(), branch)
        want = n if scaled else xh
        c, s = ck.parts()
        assert ((ref.decode(c, s, channels, code) - want).abs() <= ref.half_step(c, s, channels, code) + 2 * ROW * want.abs()).all()
    # every output on its own, no residual, no gamma
    d = B.norm_desc(rows, channels, stream, branch, eps, code, False, rx.ld, rr.ld)
    on2, ck2 = Rows(rows, channels, branch, pad, skip), Ck(rows, channels)
    B.revnet_rmsnorm_fwd(ctx, d, oh.t, None, gamma.cuda(), None, on2.t, None, None)
    assert torch.equal(on2.t, on.t)
    B.revnet_rmsnorm_fwd(ctx, d, oh.t, None, None, None, None, ck2.t, None)
    c2, s2 = ck2.parts()
    assert ((ref.decode(c2, s2, channels, code) - xh).abs() <= ref.half_step(c2, s2, channels, code) + 2 * ROW * xh.abs()).all()
    B.revnet_rmsnorm_fwd(ctx, d, rx.t, rr.t, gamma.cuda(), rx.t, None, None, None)            # in place
    assert torch.equal(rx.t, oh.t) and rx.untouched()


@pytest.mark.parametrize("source", ["h", "int8", "e4m3"])
@pytest.mark.parametrize("stream,branch", PAIRS)
@pytest.mark.parametrize("rows,channels,pad,skip", NORM_SHAPES + [(5000, 40, 0, 0), (3000, 130, 6, 0)])
def test_norm_backward(ctx, rows, channels, pad, skip, stream, branch, source):
    dn, dh, h = data(rows, channels, branch, 7), data(rows, channels, stream, 8), data(rows, channels, stream, 9)
    gamma = (1 + 0.2 * torch.randn(channels, generator=torch.Generator().manual_seed(10))).float()
    eps = 1e-5
    rstd, xh, _ = ref.norm_fwd(h.double(), gamma.double(), eps)
    ck = rs = rh = None
    if source == "h":
        rh = Rows(rows, channels, stream, pad, skip, h)
    else:
        ck = Ck.of(xh, source)
        rs = rstd.float()
        rstd, xh = rs.double(), ref.held(ck.t, rows, channels, source)
    want, dgamma = ref.norm_bwd(dn.double(), dh.double(), xh, rstd, gamma.double())
    rdn, rdh = Rows(rows, channels, branch, pad, skip, dn), Rows(rows, channels, stream, pad, skip, dh)
    dx, dr, dg = Rows(rows, channels, stream, pad, skip), Rows(rows, channels, branch, pad, skip), torch.empty(channels, device="cuda")
    d = B.norm_desc(rows, channels, stream, branch, eps, source if ck else "int8", False, rdh.ld, rdn.ld)
    ws = torch.empty(B.revnet_rmsnorm_workspace_bytes(ctx, d), dtype=torch.uint8, device="cuda")
    args = (rh.t if rh else None, ck.t if ck else None, rs.cuda() if rs is not None else None, gamma.cuda())
    B.revnet_rmsnorm_bwd(ctx, d, rdn.t, rdh.t, *args, dx.t, dr.t, dg, ws)
    gd = (dn.double() * gamma.double()).abs()
    # the mean over the row is off by ROW of the sum of magnitudes; a handful of roundings elsewhere; with h, rstd is off by ROW too
    tol = rstd[:, None] * (2 * ROW * gd + 3 * ROW * xh.abs() * (gd * xh.abs()).mean(1, keepdim=True)) + 2 * U * want.abs()
    within(dx.cpu(), want, tol, stream)
    within(dr.cpu(), want, tol, branch)
    # dgamma: a thread adds up to ceil(rows / 148) rows one after another, then up to 128 rows of a CTA, then 32 sums of up to 10 parts
    within(dg.cpu().double(), dgamma, (rows / 148 + 128 + 64) * U * (dn.double() * xh).abs().sum(0) + (ROW * (dn.double() * xh).abs().sum(0) if rh else 0))
    assert dx.untouched() and dr.untouched() and rdn.untouched()
    # without the residual's gradient, without dgamma (no workspace), in place
    dx2 = Rows(rows, channels, stream, pad, skip)
    B.revnet_rmsnorm_bwd(ctx, d, rdn.t, None, *args, dx2.t, None, None, None)
    within(dx2.cpu(), want - dh.double(), tol, stream)
    B.revnet_rmsnorm_bwd(ctx, d, rdn.t, rdh.t, *args, rdh.t, None, None, None)
    assert torch.equal(rdh.t, dx.t)
    # the same bits every time
    dg2 = torch.empty_like(dg)
    rdh2 = Rows(rows, channels, stream, pad, skip, dh)
    B.revnet_rmsnorm_bwd(ctx, d, rdn.t, rdh2.t, *args, dx2.t, None, dg2, ws)
    assert torch.equal(dg, dg2) and torch.equal(dx2.t, dx.t)

@pytest.mark.parametrize("rows,channels,pad", [(1300, 768, 0), (1300, 1280, 8), (700, 1504, 0), (1000, 2560, 8), (500, 4128, 0), (500, 5120, 0), (400, 8224, 8), (400, 12320, 0), (330, 16384, 0),
                                               (500, 1283, 3), (400, 2501, 3), (330, 5001, 3), (300, 8201, 3)])
@pytest.mark.parametrize("stream,branch", PAIRS)
def test_norm_over_many_rows(ctx, rows, channels, pad, stream, branch):
    """Threads per row, CTAs per SM and rows in shared memory go by the width; here every CTA works on several rows."""
    test_norm_forward(ctx, rows, channels, pad, 0, stream, branch, "e4m3")
    test_norm_backward(ctx, rows, channels, pad, 0, stream, branch, "int8")
    test_norm_backward(ctx, rows, channels, pad, 0, stream, branch, "h")



# ------------------------------------------------------------------ weight gradient
def wgrad(ctx, dy, ck, cin, gamma, code, dtype):
    rows, cout = dy.t.shape
    d = B.wgrad_desc(rows, cin, cout, dtype, code, dy.ld)
    ws = torch.full((B.revnet_linear_wgrad_workspace_bytes(ctx, d) + 256,), 0xFF, dtype=torch.uint8, device="cuda")     # NaN wherever it is read unwritten
    dW = torch.full((cout * cin + 8,), GUARD, device="cuda")
    B.revnet_linear_wgrad(ctx, d, dy.t, ck.t, gamma, dW[:cout * cin], ws[:-256])
    assert (dW[cout * cin:] == GUARD).all() and (ws[-256:] == 0xFF).all()
    return dW[:cout * cin].view(cout, cin).cpu().double()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout,pad,skip", [(1, 1, 1, 0, 0), (1, 64, 64, 0, 0), (63, 32, 16, 0, 0), (64, 128, 128, 0, 0), (65, 130, 40, 0, 0), (200, 257, 300, 0, 0), (129, 520, 264, 8, 0),
                                                    (1000, 96, 520, 0, 0), (700, 260, 1030, 3, 1), (2048, 512, 512, 0, 0), (4100, 72, 24, 0, 0), (513, 1000, 136, 0, 0)])
def test_weight_gradient(ctx, rows, cin, cout, pad, skip, dtype, code):
    x, dy = data(rows, cin, "f32", 11), data(rows, cout, dtype, 12)
    gamma = (1 + 0.2 * torch.randn(cin, generator=torch.Generator().manual_seed(13))).float()
    ck = Ck.of(x.double(), code, fill=0xFF)          # unwritten scale bytes: NaN if a kernel looks at them
    x8 = ref.held(ck.t, rows, cin, code)
    rdy = Rows(rows, cout, dtype, pad, skip, dy)
    got = wgrad(ctx, rdy, ck, cin, gamma.cuda(), code, dtype)
    assert rdy.untouched()
    want = dy.double().T @ x8
    size = dy.double().abs().T @ x8.abs()
    # products are exact; the tensor cores add 16 of them and the running sum with at most two steps of 2^-23 of the largest, per 16 rows (three
    # times as often where dy is float32); parts and gamma: a few roundings
    tol = (2.0 ** -22 * (rows / 16 + 1) * (3 if dtype == "f32" else 1) + 80 * U) * size
    within(got, want * gamma.double(), tol * gamma.double().abs())
    assert (got - want * gamma.double()).norm() <= 1e-5 * (want * gamma.double()).norm()
    assert torch.equal(wgrad(ctx, rdy, ck, cin, gamma.cuda(), code, dtype), got)              # the same bits every time
    within(wgrad(ctx, rdy, ck, cin, None, code, dtype), want, tol)


def test_weight_gradient_of_no_rows_and_of_single_entries(ctx):
    d = B.wgrad_desc(0, 40, 24)
    dW = torch.ones(24, 40, device="cuda")
    B.revnet_linear_wgrad(ctx, d, None, None, None, dW, None)
    assert (dW == 0).all()
    # one row, one channel at a time: every product lands where it belongs
    rows, cin, cout = 150, 300, 530
    for t, o, c in ((0, 0, 0), (149, 529, 299), (63, 128, 255), (64, 511, 256), (100, 512, 127), (127, 255, 128)):
        x, dy = torch.zeros(rows, cin, dtype=torch.float64), torch.zeros(rows, cout, dtype=torch.bfloat16)
        x[t, c], dy[t, o] = 3.0, -2.0
        got = wgrad(ctx, Rows(rows, cout, "bf16", value=dy), Ck.of(x, "int8"), cin, None, "int8", "bf16")
        assert got[o, c] == -6.0 and (got != 0).sum() == 1


def test_weight_gradient_carries_what_the_checkpoint_and_the_gradient_hold(ctx):
    """NaN blocks, infinities and NaN of the gradient reach their rows and columns of dW and no others."""
    rows, cin, cout = 100, 96, 40
    x, dy = data(rows, cin, "f32", 14), data(rows, cout, "f32", 15)
    x[10, 40], dy[20, 7], dy[30, 9] = math.nan, math.inf, math.nan
    ck = Ck.of(x.double(), "int8")
    got = wgrad(ctx, Rows(rows, cout, "f32", value=dy), ck, cin, None, "int8", "f32")
    nan = torch.zeros(cout, cin, dtype=torch.bool)
    nan[:, 32:64] = True
    nan[9] = True
    assert torch.isnan(got[nan]).all()
    rest = ~nan
    rest[7] = False
    assert torch.isfinite(got[rest]).all() and not torch.isfinite(got[7]).any()


# ------------------------------------------------------------------ log probabilities
LOGP_SHAPES = [(1, 1, 0, 0), (1, 2, 0, 0), (3, 15, 0, 0), (2, 33, 1, 1), (300, 64, 0, 0), (5, 1000, 0, 3), (40, 8191, 3, 0), (2, 32001, 0, 0), (1, 131072, 0, 0), (150, 16384, 0, 0), (9, 70000, 8, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,skip", LOGP_SHAPES)
def test_log_probabilities(ctx, rows, vocab, pad, skip, dtype):
    g = torch.Generator().manual_seed(rows + vocab)
    x = (torch.randn(rows, vocab, generator=g) * 3).to(DT[dtype])
    targets = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    if vocab > 8:
        x[0, 3:vocab // 2] = -math.inf               # masked
        targets[0] = 2
    if rows > 2:
        targets[1] = -1
        x[2] = -math.inf                             # nothing left
    r = Rows(rows, vocab, dtype, pad, skip, x)
    lse, logp, ent = ref.logprobs(x.double(), targets)
    for k in {0, 1, min(5, vocab), min(32, vocab)}:
        out = [torch.empty(rows, device="cuda") for _ in range(3)]
        tl = torch.empty(rows, k, device="cuda") if k else None
        ti = torch.empty(rows, k, dtype=torch.int32, device="cuda") if k else None
        d = B.logprob_desc(rows, vocab, dtype, k, r.ld)
        B.revnet_logprobs_fwd(ctx, d, r.t, targets.cuda(), *out, tl, ti)
        # exponents of up to |x| + |m| ~ 64 in units of log 2 are off by 2^-24 of that, ex2 by 2^-22: e-weighted sums by less; logs and the last roundings
        tol = 64 * 2.0 ** -24 + 2.0 ** -21
        within(out[0].cpu().double(), logp, tol * torch.ones_like(logp))
        within(out[1].cpu().double(), ent, 2 * tol * (1 + ent))
        within(out[2].cpu().double(), lse, tol * torch.ones_like(lse))
        assert (out[0] <= 0).all() and (out[1] >= 0).all()
        if k:
            want = ref.top(x.double(), k)
            assert torch.equal(ti.cpu(), want)
            within(tl.cpu().double(), torch.where(lse[:, None] == -math.inf, -math.inf, x.double().gather(1, want.long()) - lse[:, None]), torch.full((rows, k), tol, dtype=torch.float64))
    assert r.untouched()
    # each output on its own
    alone = torch.empty(rows, device="cuda")
    d = B.logprob_desc(rows, vocab, dtype, 0, r.ld)
    B.revnet_logprobs_fwd(ctx, d, r.t, None, None, None, alone)
    assert torch.equal(alone, out[2])


def test_ties_order_and_special_values_of_the_alternatives(ctx):
    v = 40000
    x = torch.zeros(6, v)
    x[0] = torch.arange(v).float()                   # ascending: the list changes with every logit
    x[1] = -torch.arange(v).float()
    x[2, ::7] = 1.0                                  # ties in groups
    x[3, 100], x[3, 20000], x[3, 39999] = math.nan, math.inf, -0.0
    x[4, 5:] = -math.inf
    x[5, 1::2] = -0.0                                # -0 is no less than 0
    t = torch.zeros(6, dtype=torch.int32)
    for rows in (slice(0, 6), slice(0, 1), slice(3, 4)):
        y = x[rows].cuda()
        n = y.shape[0]
        o = [torch.empty(n, device="cuda") for _ in range(3)]
        tl, ti = torch.empty(n, 20, device="cuda"), torch.empty(n, 20, dtype=torch.int32, device="cuda")
        B.revnet_logprobs_fwd(ctx, B.logprob_desc(n, v, "f32", 20), y, t[rows].cuda(), *o, tl, ti)
        assert torch.equal(ti.cpu(), ref.top(x[rows].double(), 20))
        if n == 6:
            assert torch.isnan(o[0][3]) and torch.isnan(o[1][3]) and torch.isnan(o[2][3]) and torch.isnan(tl[3]).all()
            assert torch.isfinite(torch.stack(o)[:, [0, 1, 2, 4, 5]]).all()
            assert (tl[4, 5:] == -math.inf).all()
            assert abs(o[2][5].item() - math.log(v)) < 1e-5 and abs(o[1][5].item() - math.log(v)) < 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,skip", LOGP_SHAPES)
def test_log_probability_gradient(ctx, rows, vocab, pad, skip, dtype):
    g = torch.Generator().manual_seed(7 * rows + vocab)
    x = (torch.randn(rows, vocab, generator=g) * 3).to(DT[dtype])
    targets = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    if vocab > 8:
        x[0, 3:vocab // 2] = -math.inf
        targets[0] = 2
    if rows > 2:
        targets[1] = -1
        x[2] = -math.inf
    lse, _, ent = ref.logprobs(x.double(), targets)
    lse, ent = lse.float(), ent.float()
    gl, ge = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    r = Rows(rows, vocab, dtype, pad, skip, x)
    none = (lse == -math.inf)[:, None]
    for use_g, use_e in ((True, True), (True, False), (False, True)):
        a, b = gl.double() * use_g, ge.double() * use_e
        want = ref.logprobs_bwd(x.double(), targets, lse.double(), ent.double(), a, b)
        want = torch.where(none, 0.0, want)
        q = x.double() - lse.double()[:, None]
        p = torch.exp(q)
        size = p * (a.abs()[:, None] + torch.where(p > 0, b.abs()[:, None] * (q.abs() + ent.double()[:, None]), 0.0))
        # p is off by 3 * 2^-24 |q| (the difference, the factor, its product) and ex2's 2^-22; four roundings
        tol = torch.where(none, 0.0, torch.where(p > 0, size * (3 * U * q.abs() + 2.0 ** -20), 0.0)) + 4 * U * want.abs() + 2.0 ** -126 * (1 + a.abs() + 200 * b.abs())[:, None]
        out = Rows(rows, vocab, dtype, pad, skip)
        d = B.logprob_desc(rows, vocab, dtype, 0, r.ld)
        B.revnet_logprobs_bwd(ctx, d, r.t, targets.cuda() if use_g else None, lse.cuda(), ent.cuda() if use_e else None,
                              gl.cuda() if use_g else None, ge.cuda() if use_e else None, out.t)
        hot = torch.zeros_like(want).scatter_(1, targets.clamp_min(0).long()[:, None], 1.0) * (a.abs()[:, None])
        within(out.cpu(), want, tol + 2 * U * hot, dtype)
        assert out.untouched() and r.untouched()
    B.revnet_logprobs_bwd(ctx, d, r.t, None, lse.cuda(), ent.cuda(), None, ge.cuda(), r.t)            # in place
    assert torch.equal(r.t, out.t)
    # another alignment than the logits'
    if vocab > 40:
        other = Rows(rows, vocab, dtype, pad, skip + 1)
        r2 = Rows(rows, vocab, dtype, pad, skip, x)
        B.revnet_logprobs_bwd(ctx, d, r2.t, None, lse.cuda(), ent.cuda(), None, ge.cuda(), other.t)
        assert torch.equal(other.t, out.t) and other.untouched()


def test_a_target_outside_the_vocabulary_is_reported_and_not_followed(ctx):
    x = torch.randn(3, 50).cuda()
    t = torch.tensor([3, 50, -2], dtype=torch.int32).cuda()
    o = [torch.empty(3, device="cuda") for _ in range(3)]
    B.revnet_logprobs_fwd(ctx, B.logprob_desc(3, 50, "f32"), x, t, *o)
    assert torch.isfinite(o[0][0]) and torch.isnan(o[0][1:]).all() and torch.isfinite(o[2]).all()
    with pytest.raises(B.RevnetError) as e:
        B.revnet_check_device(ctx)
    assert e.value.status == -1
    B.revnet_check_device(ctx)
    dx = torch.empty_like(x)
    B.revnet_logprobs_bwd(ctx, B.logprob_desc(3, 50, "f32"), x, t, o[2], o[1], torch.ones(3).cuda(), None, dx)
    assert torch.isfinite(dx[0]).all() and torch.isnan(dx[1:]).all()
    with pytest.raises(B.RevnetError):
        B.revnet_check_device(ctx)


# ------------------------------------------------------------------ how they are called
def test_no_rows(ctx):
    e, u8 = torch.empty(0, 32, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")
    B.revnet_act_store(ctx, B.act_desc(0, 32, "f32"), e, u8, e)
    d = B.norm_desc(0, 32, "f32", "f32")
    dg = torch.ones(32, device="cuda")
    B.revnet_rmsnorm_bwd(ctx, d, e, None, e, None, None, None, e, None, dg, torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert (dg == 0).all()
    B.revnet_logprobs_fwd(ctx, B.logprob_desc(0, 32, "f32"), e, None, None, None, None)
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits(ctx):
    """Three rows 1.2e9 elements apart: the third begins behind 2^31 elements and 2^32 bytes."""
    ld, ch = 1_200_000_001, 200
    if torch.cuda.mem_get_info()[0] < 24e9:
        pytest.skip("needs 24 GB")
    x, dy = data(3, ch, "bf16", 20), data(3, ch, "bf16", 21)
    big, big2 = (torch.empty(2 * ld + ch, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far, far2 = big.as_strided((3, ch), (ld, 1)), big2.as_strided((3, ch), (ld, 1))
    far.copy_(x)
    near = Rows(3, ch, "bf16", value=x)

    def both(call):
        outs = []
        for src, ldx in ((near.t, ch), (far, ld)):
            outs.append([t.clone() for t in call(src, ldx)])
        assert all(torch.equal(a, b) for a, b in zip(*outs))

    def store(src, ldx):
        ck, a = Ck(3, ch), Rows(3, ch, "bf16")
        B.revnet_act_store(ctx, B.act_desc(3, ch, "bf16", act="silu", ld_x=ldx), src, ck.t, a.t)
        if ldx == ld:
            B.revnet_act_store(ctx, B.act_desc(3, ch, "bf16", act="silu", ld_x=ldx, ld_a=ld), src, ck.t, far2)
            assert torch.equal(far2, a.t)
        return ck.t[:3 * 224], a.t

    def norm(src, ldx):
        n, rs = Rows(3, ch, "bf16"), torch.empty(3, device="cuda")
        B.revnet_rmsnorm_fwd(ctx, B.norm_desc(3, ch, "bf16", "bf16", ld_stream=ldx), src, None, None, None, n.t, None, rs)
        dx = Rows(3, ch, "bf16")
        B.revnet_rmsnorm_bwd(ctx, B.norm_desc(3, ch, "bf16", "bf16", ld_stream=ch, ld_branch=ldx), src, None, near.t, None, None, None, dx.t, None, None, None)
        return n.t, rs, dx.t

    def logp(src, ldx):
        o = [torch.empty(3, device="cuda") for _ in range(3)]
        t = torch.tensor([1, 2, 3], dtype=torch.int32).cuda()
        d = B.logprob_desc(3, ch, "bf16", 0, ldx)
        B.revnet_logprobs_fwd(ctx, d, src, t, *o)
        out = far2 if ldx == ld else Rows(3, ch, "bf16").t
        B.revnet_logprobs_bwd(ctx, d, src, t, o[2], o[1], o[0], o[0], out)
        return o + [out]

    def grad(src, ldx):
        d = B.wgrad_desc(3, ch, ch, "bf16", ld_dy=ldx)
        ws = torch.empty(B.revnet_linear_wgrad_workspace_bytes(ctx, d), dtype=torch.uint8, device="cuda")
        dW = torch.empty(ch, ch, device="cuda")
        B.revnet_linear_wgrad(ctx, d, src, Ck.of(dy.double(), "int8").t, None, dW, ws)
        return [dW]
    for f in (store, norm, logp, grad):
        both(f)


def test_more_rows_than_a_warp_each_can_be_counted_in_32_bits_of_threads(ctx):
    """2^27 + 100 unaligned rows: a warp for each of them makes 2^32 threads."""
    rows, ch = (1 << 27) + 100, 17
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    x = torch.empty(rows, ch, dtype=torch.bfloat16, device="cuda").normal_()
    ck = torch.empty(B.revnet_act_ckpt_bytes(ctx, rows, ch), dtype=torch.uint8, device="cuda")
    y = torch.zeros_like(x)
    d = B.act_desc(rows, ch, "bf16")
    B.revnet_act_store(ctx, d, x, ck)
    B.revnet_act_load(ctx, d, ck, y)
    for part in (slice(0, 50), slice(rows - 150, rows), slice(rows // 2, rows // 2 + 50)):
        c, s = ref.encode(x[part].cpu().double().numpy(), "int8")
        assert torch.equal(y[part].cpu().double(), ref.decode(c, s, ch, "int8"))
    assert ((y - x).abs().amax() <= x.abs().amax() / 127).item()
    n, rs = torch.zeros_like(x), torch.empty(rows, device="cuda")
    B.revnet_rmsnorm_fwd(ctx, B.norm_desc(rows, ch, "bf16", "bf16"), x, None, None, None, n, None, rs)
    for part in (slice(0, 50), slice(rows - 50, rows)):
        want, _, wn = ref.norm_fwd(x[part].cpu().double(), 1.0, 1e-5)
        within(rs[part].cpu().double(), want, ROW * want)
        within(n[part].cpu().double(), wn, (ROW + 3 * U) * wn.abs(), "bf16")


def pipeline(ctx, p, s):
    """A residual function over tokens as a user runs it: forward, loss, backward from what was kept in 8 bits.  `s` owns every buffer."""
    T, C, H, V = p["T"], p["C"], p["H"], p["V"]
    nd = B.norm_desc(T, C, "f32", "bf16", 1e-5, "int8")
    ad = B.act_desc(T, 2 * H, "bf16", "e4m3", "swiglu")
    B.revnet_rmsnorm_fwd(ctx, nd, p["x"], p["r"], p["gamma"], s["h"], s["n"], s["ck1"], s["rstd"])
    torch.matmul(s["n"], p["W1"].T, out=s["u"])
    B.revnet_act_store(ctx, ad, s["u"], s["ck2"], s["a"])
    torch.matmul(s["a"], p["W2"].T, out=s["z"])
    ld = B.logprob_desc(T, V, "bf16", 3)
    B.revnet_logprobs_fwd(ctx, ld, s["z"], p["t"], s["logp"], s["ent"], s["lse"], s["tl"], s["ti"])
    B.revnet_logprobs_bwd(ctx, ld, s["z"], p["t"], s["lse"], s["ent"], p["g"], p["ge"], s["dz"])
    torch.matmul(s["dz"], p["W2"], out=s["da"])
    B.revnet_act_bwd(ctx, ad, s["ck2"], s["da"], s["du"], s["ck3"])
    B.revnet_linear_wgrad(ctx, B.wgrad_desc(T, H, V, "bf16", "e4m3"), s["dz"], s["ck3"], None, s["dW2"], s["ws"])
    B.revnet_linear_wgrad(ctx, B.wgrad_desc(T, C, 2 * H, "bf16", "int8"), s["du"], s["ck1"], p["gamma"], s["dW1"], s["ws"])
    torch.matmul(s["du"], p["W1"], out=s["dn"])
    B.revnet_rmsnorm_bwd(ctx, nd, s["dn"], p["dh"], None, s["ck1"], s["rstd"], p["gamma"], s["dx"], s["dr"], s["dgamma"], s["ws"])


def pipeline_buffers(ctx, T, C, H, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)
    bf = torch.bfloat16
    p = dict(T=T, C=C, H=H, V=V, x=rnd(T, C), r=rnd(T, C, dtype=bf, scale=0.3), gamma=1 + rnd(C, scale=0.1), W1=rnd(2 * H, C, dtype=bf, scale=C ** -0.5),
             W2=rnd(V, H, dtype=bf, scale=2 * H ** -0.5), dh=rnd(T, C), g=rnd(T), ge=rnd(T, scale=0.1),
             t=torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32))

    def e(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")
    u8 = torch.uint8
    ws = max(B.revnet_linear_wgrad_workspace_bytes(ctx, B.wgrad_desc(T, H, V, "bf16")), B.revnet_linear_wgrad_workspace_bytes(ctx, B.wgrad_desc(T, C, 2 * H, "bf16")),
             B.revnet_rmsnorm_workspace_bytes(ctx, B.norm_desc(T, C)))
    s = dict(h=e(T, C), n=e(T, C, dtype=bf), rstd=e(T), u=e(T, 2 * H, dtype=bf), a=e(T, H, dtype=bf), z=e(T, V, dtype=bf), logp=e(T), ent=e(T), lse=e(T),
             tl=e(T, 3), ti=e(T, 3, dtype=torch.int32), dz=e(T, V, dtype=bf), da=e(T, H, dtype=bf), du=e(T, 2 * H, dtype=bf), dW1=e(2 * H, C), dW2=e(V, H),
             dn=e(T, C, dtype=bf), dx=e(T, C), dr=e(T, C, dtype=bf), dgamma=e(C), ws=e(ws, dtype=u8),
             ck1=e(B.revnet_act_ckpt_bytes(ctx, T, C), dtype=u8), ck2=e(B.revnet_act_ckpt_bytes(ctx, T, 2 * H), dtype=u8), ck3=e(B.revnet_act_ckpt_bytes(ctx, T, H), dtype=u8))
    return p, s


def rel(a, b):
    return ((a.cpu().double() - b).norm() / b.norm()).item()


def test_a_residual_function_over_tokens(ctx):
    """Forward and backward together: against the same function in float64 with the gradient that 8-bit activations give, and against exact
    gradients to the accuracy of the 8 bits."""
    T, C, H, V = 333, 264, 200, 1000
    p, s = pipeline_buffers(ctx, T, C, H, V, 31)
    pipeline(ctx, p, s)
    D = {k: v.cpu().double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in p.items()}
    t = p["t"].cpu()
    # exact: no rounding anywhere, gradients by autograd
    leaves = {k: D[k].clone().requires_grad_() for k in ("x", "W1", "W2", "gamma")}
    h = leaves["x"] + D["r"]
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-5) * leaves["gamma"]
    z = ref.act(n @ leaves["W1"].T, "swiglu") @ leaves["W2"].T
    lq = torch.log_softmax(z, 1)
    obj = (D["g"] * lq.gather(1, t.long()[:, None])[:, 0]).sum() + (D["ge"] * -(lq.exp() * lq).sum(1)).sum() + (D["dh"] * h).sum()
    gr = dict(zip(leaves, torch.autograd.grad(obj, list(leaves.values()))))
    # bf16 operands in five products (2^-9 rms each, several of them in a row) and e4m3 / int8 activations (0.03 and 0.01 rms relative)
    for got, want, tol in ((s["dx"], gr["x"], 0.05), (s["dW1"], gr["W1"], 0.06), (s["dW2"], gr["W2"], 0.06), (s["dgamma"], gr["gamma"], 0.06)):
        assert rel(got, want) < tol
    # step by step from what each step was given
    S = {k: v.cpu().double() if v.is_floating_point() else v.cpu() for k, v in s.items()}
    xh8, u8, a8 = ref.held(s["ck1"], T, C, "int8"), ref.held(s["ck2"], T, 2 * H, "e4m3"), ref.held(s["ck3"], T, H, "e4m3")
    assert rel(s["du"], ref.act_bwd(u8, S["da"], "swiglu")) < 2.0 ** -8
    assert rel(s["dW2"], S["dz"].T @ a8) < 1e-5
    assert rel(s["dW1"], (S["du"].T @ xh8) * D["gamma"]) < 1e-5
    dx, dg = ref.norm_bwd(S["dn"], D["dh"], xh8, S["rstd"], D["gamma"])
    assert rel(s["dx"], dx) < 1e-5 and rel(s["dr"], dx) < 2.0 ** -8 and rel(s["dgamma"], dg) < 1e-5
    assert torch.equal(S["ti"], ref.top(S["z"], 3))


def test_captured_calls_and_other_streams(ctx):
    """The same function on a side stream, and recorded into a graph and replayed on new inputs, two graphs on one set of streams."""
    sizes = (130, 136, 72, 500)
    sets = [pipeline_buffers(ctx, *sizes, seed) for seed in (41, 42)]
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for (p, s), st in zip(sets, side):
        with torch.cuda.stream(st):
            pipeline(ctx, p, s)
    torch.cuda.synchronize()
    keys = ("dx", "dr", "dgamma", "dW1", "dW2", "logp", "ent", "tl", "ti", "h", "ck1", "ck2", "ck3")

    def taken(s):
        out = {k: s[k].clone() for k in keys if not k.startswith("ck")}
        out["kept"] = torch.cat([ref.held(s[k], sizes[0], c, f).reshape(-1) for k, c, f in (("ck1", 136, "int8"), ("ck2", 144, "e4m3"), ("ck3", 72, "e4m3"))])
        return out
    want = [taken(s) for _, s in sets]
    graphs = []
    for p, s in sets:
        for v in s.values():
            v.view(torch.uint8).fill_(0x55)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pipeline(ctx, p, s)
        graphs.append(g)
    for _ in range(3):
        for g, st in zip(graphs, side):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for (p, s), w in zip(sets, want):
        got = taken(s)
        assert all(torch.equal(got[k], w[k]) for k in w)
    # new inputs in the recorded buffers
    sets[0][0]["x"].copy_(sets[1][0]["x"])
    for k in ("r", "gamma", "W1", "W2", "dh", "g", "ge", "t"):
        sets[0][0][k].copy_(sets[1][0][k])
    graphs[0].replay()
    torch.cuda.synchronize()
    got = taken(sets[0][1])
    assert all(torch.equal(got[k], want[1][k]) for k in got)
    del graphs


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("mode,frac,split,cin,k,stride", [(0, 16, 1, 64, 3, 2), (0, 0, 1, 24, 1, 1), (1, 0, 0, 20, 3, 1), (0, 12, 0, 32, 3, 2), (1, 16, 1, 8, 1, 2)])
def test_stored_layer_from_its_kept_input(ctx, mode, frac, split, cin, k, stride, code):
    """revnet_transition_bwd_kept has the bits of revnet_transition_bwd on the values that were kept, and these are the format's."""
    N, H, cout = 3, 10, 32
    d = B.TransitionDesc(N, H, H, cin, cout, k, stride, split, 1e-5, mode, frac)
    g = torch.Generator().manual_seed(cin + k)
    halves, c = (2, cin // 2) if split else (1, cin)
    x = [torch.randn(N * H * H, c, generator=g) * 2 for _ in range(halves)]
    fixed = frac and split           # (a plain input is float32 whatever the state's format)
    raw = [torch.round(t.double() * 2 ** frac).to(torch.int32) if fixed else t for t in x]
    val = [t.double() / 2 ** frac if fixed else t.double() for t in raw]
    dev = [t.cuda() for t in raw] + [None] * (2 - halves)
    kept_bytes, ws_bytes = B.revnet_transition_kept_bytes(ctx, d)
    kept = torch.full((kept_bytes,), 0xA5, dtype=torch.uint8, device="cuda")
    B.revnet_transition_keep(ctx, d, *dev, code, kept)
    part = kept_bytes // halves
    x8 = []
    for i, t in enumerate(val):
        wc, ws = ref.encode(t.float().double().numpy(), code)
        gc, gs = ref.take_apart(kept[i * part:], N * H * H, c)
        assert (gs == ws).all() and (ref.code_values(gc, code) == ref.code_values(wc, code)).all()
        x8.append(ref.decode(wc, ws, c, code).float().cuda())
    W = (torch.randn(cout, k, k, cin, generator=g) * (2 / (cin * k * k)) ** 0.5).cuda()
    gamma, beta = (1 + 0.1 * torch.randn(cin, generator=g)).cuda(), (0.1 * torch.randn(cin, generator=g)).cuda()
    out = N * (-(-H // stride)) ** 2
    dout = [torch.randn(out, cout // 2, generator=g).cuda() for _ in range(2)]

    def grads():
        return [torch.empty(N * H * H, c, device="cuda") for _ in range(halves)] + [None] * (2 - halves) + [torch.empty_like(W), torch.empty_like(gamma), torch.empty_like(beta)]
    got, want = grads(), grads()
    B.revnet_transition_bwd_kept(ctx, d, code, kept, *dout, W, gamma, beta, *got, torch.empty(ws_bytes, dtype=torch.uint8, device="cuda"))
    f = B.TransitionDesc(N, H, H, cin, cout, k, stride, split, 1e-5, mode, 0)
    ws = torch.empty(B.revnet_transition_workspace_bytes(ctx, f)[1], dtype=torch.uint8, device="cuda")
    B.revnet_transition_bwd(ctx, f, *(x8 + [None] * (2 - halves)), *dout, W, gamma, beta, *want, ws)
    for a, b in zip(got, want):
        assert a is None or torch.equal(a, b)


def test_refusals_on_the_device(ctx):
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    ck = Ck(4, 64)
    for bad in (x[:, :32], x.t().contiguous().t(), x.float(), x.cpu(), x[:3]):
        with pytest.raises(B.RevnetError, match="x must be"):
            B.revnet_act_store(ctx, B.act_desc(4, 64), bad, ck.t)
    with pytest.raises(B.RevnetError, match="ck must hold"):
        B.revnet_act_store(ctx, B.act_desc(4, 64), x, ck.t[:-1])
    with pytest.raises(B.RevnetError) as e:
        B.revnet_act_store(ctx, B.act_desc(4, 64), x, ck.buf[16:16 + ck.n])
    assert e.value.status == -4
    d = B.wgrad_desc(4, 64, 64)
    with pytest.raises(B.RevnetError) as e:
        B.revnet_linear_wgrad(ctx, d, x, ck.t, None, torch.empty(64, 64, device="cuda"), torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -3


# ------------------------------------------------------------------ calls that skip ctypes
def every_call(ctx):
    """One call of each entry point -> what they wrote."""
    rows, c = 9, 64
    x, r, dn = (data(rows, c, "f32", i).cuda() for i in (41, 42, 43))
    gamma, rstd, dg = torch.ones(c, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(c, device="cuda")
    h, n, dx, dr, a, da = (torch.zeros(rows, c, device="cuda") for _ in range(6))
    ck, ack = Ck(rows, c), Ck(rows, c)
    d = B.norm_desc(rows, c, "f32", "f32")
    ws = torch.zeros(B.revnet_rmsnorm_workspace_bytes(ctx, d), dtype=torch.uint8, device="cuda")
    B.revnet_rmsnorm_fwd(ctx, d, x, r, gamma, h, n, ck.t, rstd)
    B.revnet_rmsnorm_bwd(ctx, d, dn, None, None, ck.t, rstd, gamma, dx, dr, dg, ws)
    e = B.act_desc(rows, c, "f32", act="silu")
    B.revnet_act_load(ctx, e, ck.t, a)
    B.revnet_act_bwd(ctx, e, ck.t, dn, da, ack.t)
    dW, kept = torch.empty(c, c, device="cuda"), Ck(rows, c)
    B.revnet_act_store(ctx, e, x, kept.t)
    f = B.wgrad_desc(rows, c, c, "f32")
    ws2 = torch.zeros(B.revnet_linear_wgrad_workspace_bytes(ctx, f), dtype=torch.uint8, device="cuda")
    B.revnet_linear_wgrad(ctx, f, dn, kept.t, None, dW, ws2)
    g = B.logprob_desc(rows, c, "f32", 3)
    logp, entropy, lse = (torch.empty(rows, device="cuda") for _ in range(3))
    top, index, targets, dl = torch.empty(rows, 3, device="cuda"), torch.empty(rows, 3, dtype=torch.int32, device="cuda"), torch.arange(rows, dtype=torch.int32, device="cuda"), torch.empty_like(x)
    B.revnet_logprobs_fwd(ctx, g, x, targets, logp, entropy, lse, top, index)
    B.revnet_logprobs_bwd(ctx, g, x, targets, lse, entropy, logp, None, dl)
    return [h, n, rstd, dx, dr, dg, a, da, dW, ack.t, kept.t, logp, entropy, lse, top, index, dl]


def test_direct_calls_do_what_the_checked_ones_do(ctx, monkeypatch):
    assert B._direct is not None
    with monkeypatch.context() as m:
        m.setattr(B, "_direct", None)
        want = every_call(ctx)

    def unused(*a):
        raise AssertionError("the direct call was not taken")
    for name in ("_row_ptr", "_flat_ptr", "_ck_ptr", "_ws", "_stream_of"):
        monkeypatch.setattr(B, name, unused)
    assert all(torch.equal(a, b) for a, b in zip(every_call(ctx), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):     # on the stream that is current
        got = every_call(ctx)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_direct_calls_leave_refusals_to_the_checked_ones(ctx):
    d, x, ck = B.act_desc(4, 64, "f32"), torch.zeros(4, 64, device="cuda"), Ck(4, 64)
    call = lambda *a: B._direct.act_store(ctx.h.value, ctx.device, *a)
    assert call(d, x, ck.t, None) == 0
    for bad in (x[:, :63], x.double(), x.cpu(), x.t(), x.bfloat16(), x[:3], x.view(-1), x.to_sparse(), "x", 5, x.expand(2, 4, 64)):
        assert call(d, bad, ck.t, None) is None
    assert call(d, x, ck.t[:-1], None) is None and call(d, x, ck.t.to(torch.int8), None) is None and call(d, x, ck.t) is None
    assert call(B.logprob_desc(4, 64, "f32"), x, ck.t, None) is None and call(None, x, ck.t, None) is None
    assert B._direct.act_store(0, ctx.device, d, x, ck.t, None) is None and B._direct.act_store(ctx.h.value, ctx.device + 1, d, x, ck.t, None) is None
    assert B._direct.act_store(None, ctx.device, d, x, ck.t, None) is None
    with pytest.raises(B.RevnetError, match="x must be"):
        B.revnet_act_store(ctx, d, x.double(), ck.t)
    with pytest.raises(B.RevnetError) as e:              # what only the entry point refuses
        B.revnet_act_store(ctx, B.act_desc(4, 63, "f32", act="swiglu"), torch.zeros(4, 63, device="cuda"), Ck(4, 63).t)
    assert e.value.status < 0
    torch.cuda.synchronize()
