"""Operators on rows of tokens at values where float32's range or resolution ends, against float64.  Tolerances are bounds on rounding errors, as in
test_gpu_token_rows.py."""
import math

import pytest
import torch

from paper_1707_04585_b200 import binding as B
from tests import token_ref as ref
from tests.test_gpu_token_rows import Ck, Rows, data, wgrad, within
from tests.token_ref import DT, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    B.revnet_check_device(c)
    c.close()


# ------------------------------------------------------------------ log probabilities of large finite logits
def large_logits(vocab, dtype, seed=1):
    """Rows by name: masks of the type's lowest value and of round numbers, the largest values, and values whose differences are small beside them."""
    g = torch.Generator().manual_seed(seed)
    lo, hi = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max

    def normal():
        return torch.randn(vocab, generator=g) * 3

    def full(v):
        return torch.full((vocab,), float(v))

    def mixed(*parts):               # the parts' values by turns
        t = torch.stack([p if torch.is_tensor(p) else full(p) for p in parts])
        return t[torch.arange(vocab) % len(parts), torch.arange(vocab)]

    def with_one(t, v, at=None):
        t = t.clone()
        t[vocab // 3 if at is None else at] = v
        return t
    near = torch.rand(vocab, generator=g) * 4 - 2
    rows = dict(all_lowest=full(lo), all_largest=full(hi), half_lowest=mixed(lo, normal()), lowest_and_none=mixed(lo, -math.inf), one_left=with_one(full(lo), -3.0),
                one_large=with_one(normal(), 2.5e38), one_largest=with_one(normal(), hi, vocab - 1), two_large=with_one(with_one(normal(), 3e38), 3e38, 0),
                all_5e9=full(-5e9), all_1e10=full(1e10), masked_1e10=mixed(-1e10, normal(), normal()), all_masks=mixed(-1e9, -1e10, lo), all_1e30=full(-1e30), both_signs=mixed(-1e30, 1e30),
                around_million=near + 2.0 ** 20, around_minus_million=near - 2.0 ** 20, thousands=near - 3000.0, growing=torch.linspace(-88, 88, vocab).double().exp().float() * 4,
                shrinking=-torch.linspace(-88, 88, vocab).double().exp().float().flip(0) * 4, falling=torch.linspace(88, -88, vocab).double().exp().float() * 4,       # (to +inf: NaN)
                growing_finite=torch.linspace(-88, 88, vocab).double().exp().float() * 2, falling_finite=torch.linspace(88, -88, vocab).double().exp().float() * 2)
    return list(rows), torch.stack(list(rows.values())).to(DT[dtype])


def definition(x, targets):
    """Float64 -> (lse, logp of the targets, entropy, log p of every logit): in differences from the maximum, since lse alone has no room for log s beside 1e38."""
    m = x.amax(1, keepdim=True)
    logs = torch.log(torch.exp(x - m).sum(1, keepdim=True))
    q = (x - m) - logs
    p = torch.exp(q)
    ent = -torch.where(p == 0, 0.0, p * q).sum(1)
    return (m + logs)[:, 0], torch.where(targets < 0, 0.0, q.gather(1, targets.clamp_min(0).long()[:, None])[:, 0]), ent, q


def forward(ctx, r, targets, vocab, dtype, k):
    n = r.t.shape[0]
    out = [torch.empty(n, device="cuda") for _ in range(3)]
    tl = torch.empty(n, k, device="cuda") if k else None
    ti = torch.empty(n, k, dtype=torch.int32, device="cuda") if k else None
    B.revnet_logprobs_fwd(ctx, B.logprob_desc(n, vocab, dtype, k, r.ld), r.t, targets.cuda(), *out, tl, ti)
    return out, tl, ti


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,pad,repeat", [(5, 0, 1), (1000, 0, 1), (1003, 3, 1), (40000, 0, 1), (4099, 0, 60), (131072, 0, 0)])
def test_log_probabilities_of_large_logits(ctx, vocab, pad, repeat, dtype):
    """One row per CTA, rows cut over a cluster (few of them), a single row at a time."""
    names, x = large_logits(vocab, dtype)
    g = torch.Generator().manual_seed(vocab)
    targets = torch.randint(0, vocab, (len(names),), generator=g, dtype=torch.int32)
    targets[names.index("one_large")] = vocab // 3
    lse, logp, ent, q = definition(x.double(), targets)
    # exponents (x - m) log2 e are off by 2 * 2^-24 of themselves, and beyond 32 of them the weight is below 2^-32; ex2 by 2^-22; logs and last roundings
    tol = 64 * 2.0 ** -24 + 2.0 ** -21
    for rows in [slice(i, i + 1) for i in range(len(names))] if repeat == 0 else [slice(None)]:
        n = max(repeat, 1)
        xs, ts = x[rows].repeat(n, 1), targets[rows].repeat(n)
        r = Rows(xs.shape[0], vocab, dtype, pad, 0, xs)
        for k in (0, min(5, vocab)):
            out, tl, ti = forward(ctx, r, ts, vocab, dtype, k)
            within(out[0].cpu().double(), logp[rows].repeat(n), tol * torch.ones(xs.shape[0], dtype=torch.float64))
            within(out[1].cpu().double(), ent[rows].repeat(n), 2 * tol * (1 + ent[rows].repeat(n)))
            within(out[2].cpu().double(), lse[rows].repeat(n), tol * torch.ones(xs.shape[0], dtype=torch.float64))
            if k:
                want = ref.top(x[rows].double(), k)
                assert torch.equal(ti.cpu(), want.repeat(n, 1))
                within(tl.cpu().double(), q[rows].gather(1, want.long()).repeat(n, 1), torch.full((xs.shape[0], k), tol, dtype=torch.float64))


@pytest.mark.parametrize("vocab", [40, 3000, 70000])
def test_bad_logits_among_large_ones_stay_bad(ctx, vocab):
    x = torch.full((6, vocab), torch.finfo(torch.float32).min)
    x[0, 7], x[1, vocab - 1], x[2] = math.nan, math.inf, -math.inf
    x[3], x[3, 2] = -math.inf, math.nan
    x[4], x[4, 5] = torch.finfo(torch.float32).max, math.nan
    x[5], x[5, 9] = torch.finfo(torch.float32).max, math.inf
    out, tl, ti = forward(ctx, Rows(6, vocab, "f32", value=x), torch.zeros(6, dtype=torch.int32), vocab, "f32", 3)
    bad = torch.tensor([True, True, False, True, True, True])
    for o in out:
        assert torch.isnan(o.cpu()[bad]).all()
    assert out[0][2] == -math.inf and out[1][2] == 0 and out[2][2] == -math.inf and (tl[2] == -math.inf).all()
    assert torch.equal(ti.cpu(), ref.top(x.double(), 3))


def gradient(ctx, r, targets, lse, ent, gl, ge, out):
    n, vocab = r.t.shape
    dtype = "f32" if r.t.dtype == torch.float32 else "bf16"
    B.revnet_logprobs_bwd(ctx, B.logprob_desc(n, vocab, dtype, 0, r.ld), r.t, targets.cuda(), lse, ent, gl.cuda(), ge.cuda() if ge is not None else None, out.t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,pad,repeat", [(5, 0, 1), (1000, 0, 1), (1003, 3, 1), (70000, 0, 1), (4099, 0, 60), (200000, 0, 1)])
def test_gradient_of_large_logits(ctx, vocab, pad, repeat, dtype):
    """From the lse and entropy that the forward call gave, which float32 holds to 2^-24 of lse only: rows where that is coarse are summed again."""
    names, x = large_logits(vocab, dtype)
    keep = torch.isfinite(x.double().amax(1))                    # (rows with +inf are NaN)
    x = x[keep].repeat(repeat, 1)
    n = x.shape[0]
    g = torch.Generator().manual_seed(vocab + 1)
    targets = torch.randint(-1, vocab, (n,), generator=g, dtype=torch.int32)
    gl, ge = torch.randn(n, generator=g), torch.randn(n, generator=g)
    r = Rows(n, vocab, dtype, pad, 0, x)
    (logp, ent, lse), _, _ = forward(ctx, r, targets, vocab, dtype, 0)
    lse64, _, ent64, q = definition(x.double(), targets)
    p = torch.exp(q)
    live = torch.where(targets < 0, 0.0, gl.double())[:, None]
    hot = torch.zeros_like(q).scatter_(1, targets.clamp_min(0).long()[:, None], 1.0) * live
    for b in (None, ge):
        w = b.double()[:, None] if b is not None else 0.0
        bent = torch.where(p > 0, q + ent64[:, None], 0.0)
        want = hot - p * (live + w * bent)
        size = p * (live.abs() + (w.abs() if b is not None else 0.0) * torch.where(p > 0, q.abs() + ent64[:, None], 0.0))
        # q is off by what float32 keeps of lse (up to 4096; beyond, log s is kept apart), by 3 * 2^-24 of itself (the difference, the factor, its product) and
        # by log s's 2^-21; ex2 by 2^-22; the entropy by the forward's tolerance; a few roundings
        dq = 3 * U * q.abs() + U * lse64.abs().clamp_max(4096)[:, None] + 2.0 ** -20
        dent = ((64 * 2.0 ** -24 + 2.0 ** -21) * 2 * (1 + ent64) + U * ent64)[:, None]
        tol = torch.where(p > 0, size * dq + p * (w.abs() if b is not None else 0.0) * (dq + dent) + 8 * U * size, 0.0) + 2.0 ** -126 * (1 + live.abs() + 200 * (w.abs() if b is not None else 0.0)) + 2 * U * hot.abs()
        out = Rows(n, vocab, dtype, pad)
        gradient(ctx, r, targets, lse, ent if b is not None else None, gl, b, out)
        within(out.cpu(), want, tol, dtype)
        assert out.untouched()
        again = Rows(n, vocab, dtype, pad, 0, x)                 # in place: every part of a row has to see all of it before any is overwritten
        gradient(ctx, again, targets, lse, ent if b is not None else None, gl, b, again)
        assert torch.equal(again.t, out.t) and again.untouched()


@pytest.mark.parametrize("size,vocab", [(1e4, 3000), (1e6, 50000)])
def test_gradient_of_a_part_of_a_vocabulary_takes_the_given_lse(ctx, size, vocab):
    """lse of more logits than the call sees: it is taken as it is, however coarse."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(4, vocab, generator=g) + size
    rest = torch.full((4, 1), float(size + 20 * max(1.0, size * 2.0 ** -20)))      # one more logit, far above
    lse = torch.logsumexp(torch.cat([x, rest], 1).double(), 1).float()
    targets, gl = torch.tensor([0, 5, -1, vocab - 1], dtype=torch.int32), torch.randn(4, generator=g)
    r, out = Rows(4, vocab, "f32", value=x), Rows(4, vocab, "f32")
    gradient(ctx, r, targets, lse.cuda(), None, gl, None, out)
    want = ref.logprobs_bwd(x.double(), targets, lse.double(), torch.zeros(4, dtype=torch.float64), gl.double(), torch.zeros(4, dtype=torch.float64))
    q = x.double() - lse.double()[:, None]
    hot = torch.zeros_like(want).scatter_(1, targets.clamp_min(0).long()[:, None], 1.0) * gl.double().abs()[:, None]
    within(out.cpu(), want, torch.exp(q) * gl.double().abs()[:, None] * (3 * U * q.abs() + 2.0 ** -20) + 2.0 ** -126 + 2 * U * hot)


# ------------------------------------------------------------------ weight gradients over many rows
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", [(1000, 96, 136), (2048, 4096, 4096), (16500, 2048, 1280), (66000, 1530, 1790)])
def test_weight_gradient_of_many_rows_of_one_sign(ctx, rows, cin, cout, dtype):
    """The tensor cores cut their running sum off after every 16 rows.  With operands of one sign that is a bias, half a step of 2^-23 on average; a run of
    1024 rows has 64 of them, of a sum that is half the run's on average, whatever the number of runs.  (Tiles enough for shares of several runs.)"""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cin, device="cuda", generator=g).abs()
    dy = torch.randn(rows, cout, device="cuda", generator=g).abs().to(DT[dtype])
    ck, x8 = Ck(rows, cin), torch.empty(rows, cin, device="cuda")
    B.revnet_act_store(ctx, B.act_desc(rows, cin, "f32"), x, ck.t)
    B.revnet_act_load(ctx, B.act_desc(rows, cin, "f32"), ck.t, x8)
    got = wgrad(ctx, Rows(rows, cout, dtype, value=dy), ck, cin, None, "int8", dtype).cuda()
    want = dy.double().T @ x8.double()
    err = (got - want) / want
    assert abs(err.mean()) <= 64 / 2 / 2 * 2.0 ** -23
    # at most two steps each time, and a rounding per run and part
    assert err.abs().max() <= 64 / 2 * 2.0 ** -22 + (rows / 1024 + 80) * U


def schedule(rows, cin, cout, parts, sms):
    """How the kernel deals out its tiles (csrc/wgrad8.cu): whole tiles per pair, tiles left over, pairs that share those, whether a pair's share goes on from one
    tile into the next."""
    steps, most = -(-rows // 64) * parts, min(sms // 2, 80)
    tiles = -(-cin // 256) * -(-cout // 256)

    def sharers_of(t):
        return min(max(t, -(-t * steps // 8)), most)
    pairs = sharers_of(tiles)
    if tiles < pairs and steps - tiles * steps // pairs < 32:
        pairs = tiles
    waves = tiles // pairs
    rest = tiles - waves * pairs
    sharers = sharers_of(rest) if rest else 0
    if rest and steps - rest * steps // sharers < 32:
        sharers = rest
    elif rest and sharers // rest * rest >= sharers * 85 // 100:
        sharers -= sharers % rest
    begin = [rest * steps * q // sharers for q in range(sharers + 1)] if sharers else []
    crossing = any(a // steps != (b - 1) // steps for a, b in zip(begin, begin[1:]))
    split = rest > 0 and rest % sharers != 0
    return waves, rest, sharers, crossing, split


# rows, input and output channels; whole tiles per pair, whether tiles are cut, whether a share crosses from one into the next (148 SMs)
SCHEDULES = [(4096, 1280, 1024, 0, True, True), (8192, 2560, 1000, 0, True, True), (4096, 4096, 4096, 3, True, False), (4096, 500, 12032, 1, True, True),
             (8100, 1530, 4860, 1, True, True), (64, 4096, 5120, 4, False, False), (100, 2049, 10000, 4, False, False)]


@pytest.mark.parametrize("dtype,code", [("bf16", "int8"), ("bf16", "e4m3"), ("f32", "int8")])
@pytest.mark.parametrize("rows,cin,cout,waves,cut,crossing", SCHEDULES)
def test_weight_gradient_schedules(ctx, rows, cin, cout, waves, cut, crossing, dtype, code):
    """Pairs with several whole tiles, tiles cut into parts behind them, shares that cross from one tile into the next."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    if dtype == "f32":
        rows = rows // 3             # (three products: about the same schedule)
    got_waves, rest, sharers, got_crossing, got_cut = schedule(rows, cin, cout, 3 if dtype == "f32" else 1, sms)
    if sms == 148 and dtype == "bf16":
        assert (got_waves, got_cut, got_crossing) == (waves, cut, crossing)
    ld = -(-cout // 8) * 8
    d = B.wgrad_desc(rows, cin, cout, dtype, code, ld)
    prepared = 0 if dtype == "bf16" else -(-(-(-rows // 64) * 3 * 64 * ld * 2) // 256) * 256
    assert B.revnet_linear_wgrad_workspace_bytes(ctx, d) == prepared + (sharers * 2 * 65536 * 4 if got_cut else 0) + 256
    x, dy = data(rows, cin, "f32", 23), data(rows, cout, dtype, 24)
    ck = Ck.of(x.double(), code, fill=0xFF)
    rdy = Rows(rows, cout, dtype, ld - cout, 0, dy)
    got = wgrad(ctx, rdy, ck, cin, None, code, dtype).cuda()
    x8, dy64 = ref.held(ck.t, rows, cin, code).cuda(), dy.double().cuda()
    want, size = dy64.T @ x8, dy64.abs().T @ x8.abs()
    # as in test_weight_gradient, runs of 1024 rows: two steps of 2^-23 every 16 rows of at most a run, a rounding per run and part
    tol = (2.0 ** -22 * (min(rows, 1024) / 16 + 1) * (3 if dtype == "f32" else 1) + (rows / 1024 + 80) * U) * size
    assert ((got - want).abs() <= tol + U * want.abs()).all()
    assert rdy.untouched()


# ------------------------------------------------------------------ activations far out
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("kind", ["gelu", "silu", "swiglu", "relu"])
def test_activations_of_the_largest_values(ctx, kind, code):
    """Out there an activation is x or 0 and its derivative 1 or 0; sums and products on the way stay finite or their limits are taken."""
    sizes = [20.0, 1e4, 1e9, 1e13, 1.1e19, 3e19, 1e20, 1e30, 3e38]
    x = torch.tensor([[s, -s] * 16 for s in sizes])              # one block per row: every value is held to its code's step
    if kind == "swiglu":
        x = torch.cat([x, torch.full_like(x, 0.5)], 1)           # gates of all sizes, and what they gate
    rows, c = x.shape
    out = c // 2 if kind == "swiglu" else c
    ck, a = Ck(rows, c), Rows(rows, out, "f32")
    d = B.act_desc(rows, c, "f32", code, kind)
    B.revnet_act_store(ctx, d, x.cuda(), ck.t, a.t)
    x8 = ref.held(ck.t, rows, c, code)
    first = x[:, :out]
    up = 0.5 if kind == "swiglu" else 1.0
    within(a.cpu(), torch.where(first > 0, first.double() * up, 0.0), 2.0 ** -20 * first.double().abs().clamp_max(1e4) * up)      # (20 is not quite there: e^-20 20 = 4e-8)
    da, dx, ack = torch.full((rows, out), 3.0), Rows(rows, c, "f32"), Ck(rows, out)
    B.revnet_act_bwd(ctx, d, ck.t, da.cuda(), dx.t, ack.t)
    g8 = x8[:, :out]
    within(dx.cpu()[:, :out], torch.where(g8 > 0, 3.0 * up, 0.0).double(), torch.full_like(g8, 2.0 ** -18))
    if kind == "swiglu":
        want = torch.where(g8 > 0, 3.0 * g8, 0.0)
        within(dx.cpu()[:, out:], torch.where(want > torch.finfo(torch.float32).max, math.inf, want), 2.0 ** -20 * g8.abs().clamp_max(1e4))      # (3 * 3e38 is beyond float32)
    assert torch.isfinite(ref.held(ack.t, rows, out, code)).all()


# ------------------------------------------------------------------ what lies between rows
@pytest.mark.parametrize("stream,branch", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,channels,pad,skip", [(300, 45, 2, 1), (700, 1001, 3, 5), (200, 5001, 1, 7), (90, 8203, 5, 3)])
def test_what_lies_between_rows_changes_nothing(ctx, rows, channels, pad, skip, stream, branch):
    """Infinities and NaN in front of the first row, between the rows and behind the last one."""
    x, r, dn, dh = (data(rows, channels, t, i) for i, t in enumerate((stream, branch, branch, stream)))
    gamma = torch.ones(channels).cuda()
    got = []
    for fill in (0.0, math.inf, math.nan):
        def view(t, dtype):
            v = Rows(rows, channels, dtype, pad, skip, t)
            v.buf[v.out] = fill
            return v
        vx, vr, vdn, vdh = view(x, stream), view(r, branch), view(dn, branch), view(dh, stream)
        h, n, ck, rstd = Rows(rows, channels, stream, pad, skip), Rows(rows, channels, branch, pad, skip), Ck(rows, channels), torch.empty(rows, device="cuda")
        d = B.norm_desc(rows, channels, stream, branch, 1e-5, "int8", False, vx.ld, vr.ld)
        B.revnet_rmsnorm_fwd(ctx, d, vx.t, vr.t, gamma, h.t, n.t, ck.t, rstd)
        dx, dg = Rows(rows, channels, stream, pad, skip), torch.empty(channels, device="cuda")
        ws = torch.empty(B.revnet_rmsnorm_workspace_bytes(ctx, d), dtype=torch.uint8, device="cuda")
        B.revnet_rmsnorm_bwd(ctx, d, vdn.t, vdh.t, None, ck.t, rstd, gamma, dx.t, None, dg, ws)
        da, a = Rows(rows, channels, branch, pad, skip), Rows(rows, channels, branch, pad, skip)
        e = B.act_desc(rows, channels, branch, "int8", "silu", vr.ld, vr.ld)
        kept = Ck(rows, channels)
        B.revnet_act_store(ctx, e, vr.t, kept.t, a.t)
        B.revnet_act_bwd(ctx, e, kept.t, vdn.t, da.t)
        got.append([t.clone() for t in (h.t, n.t, rstd, dx.t, dg, a.t, da.t)])
    for other in got[1:]:
        assert all(torch.equal(p, q) for p, q in zip(got[0], other)) and all(torch.isfinite(p.float()).all() for p in other)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_whose_squares_leave_the_range_of_float32(ctx, dtype):
    """Such a row has rstd 0, and nothing of it is kept; the others are as ever."""
    x = data(4, 300, dtype, 30)
    x[1], x[2, 7] = 1e19, -3e38
    n, rstd, ck = Rows(4, 300, dtype), torch.empty(4, device="cuda"), Ck(4, 300)
    B.revnet_rmsnorm_fwd(ctx, B.norm_desc(4, 300, dtype, dtype), x.cuda(), None, None, None, n.t, ck.t, rstd)
    want, _, wn = ref.norm_fwd(x.double(), 1.0, 1e-5)
    assert (rstd[1:3] == 0).all() and (n.t[1:3] == 0).all() and (ref.held(ck.t, 4, 300, "int8")[1:3] == 0).all()
    for i in (0, 3):
        within(rstd.cpu().double()[i:i + 1], want[i:i + 1], 64 * U * want[i:i + 1])
        within(n.cpu()[i], wn[i], 67 * U * wn[i].abs(), dtype)
