"""The token-row operators of this library as cases that can be timed and compared with their plain forms.

Rows are tokens (or pixels), channels are contiguous.  Activations kept for the backward pass in 8 bits ("checkpoints") hold one
byte per value, int8 or e4m3, and a power-of-two scale per 32 consecutive channels of a row:

  codes   [rows][pitch], pitch = channels rounded up to 32, zeros behind the last channel
  scales  [ceil(channels / 128)][rows rounded up to 64][4] bytes e + 127, at the next multiple of 256 bytes behind the codes

with e the least integer (at least -117) for which the largest magnitude of the 32 is <= 127 * 2^e (int8) or 448 * 2^e (e4m3), and the
code value * 2^-e rounded to nearest, ties to even.  A block with an infinity or a NaN has byte 255 and codes 0, and decodes to NaN.

  op         what one pass is
  norm_fwd   h = x + r, its root-mean-square norm n = h / rms(h) * gamma, the normalised rows h / rms(h) kept in 8 bits and read back
  norm_bwd   the gradients of that from the kept rows ("ck") or from h ("h"), with the gradient that reaches h from the residual path
  act_fwd    an activation function and its input kept in 8 bits, read back
  act_bwd    its backward pass from the kept input, the activation recomputed and kept in 8 bits for the next weight gradient, read back
  wgrad      the weight gradient of a linear layer whose normalised input was kept in 8 bits
  logp_fwd   log probabilities of given tokens, entropy and the k most likely alternatives of each row of logits
  logp_bwd   the gradient of the log probabilities and entropies with respect to the logits
"""
import math

import torch

own = False

EPS = 1e-5
GROUP = 32
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
TOP = {"int8": 127.0, "e4m3": 448.0}
CK = 1 + 1 / GROUP          # bytes per value of a checkpoint


# ------------------------------------------------------------------ the cases
def _norm_fwd(rows, channels, stream, branch, fmt, res=True, pad=0):
    return dict(op="norm_fwd", rows=rows, channels=channels, stream=stream, branch=branch, fmt=fmt, res=res, pad=pad)


def _norm_bwd(rows, channels, stream, branch, fmt, source, pad=0):
    return dict(op="norm_bwd", rows=rows, channels=channels, stream=stream, branch=branch, fmt=fmt, source=source, pad=pad)


def _act(op, rows, channels, dtype, fmt, act, pad=0):
    return dict(op=op, rows=rows, channels=channels, dtype=dtype, fmt=fmt, act=act, pad=pad)


def _wgrad(rows, cin, cout, dtype, fmt, gamma=True, pad=0):
    return dict(op="wgrad", rows=rows, cin=cin, cout=cout, dtype=dtype, fmt=fmt, gamma=gamma, pad=pad)


def _logp(op, rows, vocab, dtype, k, masked=False, pad=0):
    return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, k=k, masked=masked, pad=pad)


def listed():
    return [
        # one token on its way through a layer while text is generated: latency
        dict(_norm_fwd(1, 4096, "bf16", "bf16", "int8"), name="norm_fwd_token"),
        # a layer's norm over a training batch of eight sequences of 2048 tokens, everything in bf16
        dict(_norm_fwd(16384, 4096, "bf16", "bf16", "int8"), name="norm_fwd_train"),
        # the backward of a norm in front of a branch of the first stage of the large-image network: 64 images of 56 x 56 pixels,
        # 512 channels, float32 coupling state, bf16 branch, from the 8-bit rows
        dict(_norm_bwd(64 * 56 * 56, 512, "f32", "bf16", "int8", "ck"), name="norm_bwd_image"),
        # the same in single precision on a ragged batch whose rows are not aligned, from the residual stream itself
        dict(_norm_bwd(777, 1001, "f32", "f32", "e4m3", "h"), name="norm_bwd_odd"),
        # the gated activation between the two linear layers of a wide token function
        dict(_act("act_fwd", 16384, 16384, "bf16", "int8", "swiglu"), name="act_fwd_gated"),
        dict(_act("act_bwd", 16384, 16384, "bf16", "int8", "swiglu"), name="act_bwd_gated"),
        # a small ungated function in single precision, odd batch, rows inside a wider buffer
        dict(_act("act_bwd", 999, 1000, "f32", "e4m3", "gelu", 24), name="act_bwd_odd"),
        # weight gradient of a square linear layer over the training batch
        dict(_wgrad(16384, 4096, 4096, "bf16", "int8"), name="wgrad_train"),
        # the same with single-precision gradients, ragged in every direction
        dict(_wgrad(1999, 520, 1000, "f32", "e4m3"), name="wgrad_odd"),
        # the loss of a training batch over a large vocabulary, and its gradient
        dict(_logp("logp_fwd", 4096, 131072, "bf16", 0), name="logp_fwd_train"),
        # scoring eight sequences' next tokens with their alternatives, padded vocabulary of odd length
        dict(_logp("logp_fwd", 8, 128001, "f32", 20, True), name="logp_fwd_score"),
        dict(_logp("logp_bwd", 4096, 50000, "bf16", 0), name="logp_bwd_train"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "act_fwd", "act_bwd", "wgrad", "logp_fwd", "logp_bwd"])
    fmt = rng.choice(["int8", "e4m3"])
    pad = rng.choice([0, 0, 0, 8, 3])
    if op.startswith("norm"):
        channels = _log(rng, 16, 8192)
        channels = channels if rng.random() < 0.3 else max(16, channels // 32 * 32)
        rows = _log(rng, 1, min(1 << 17, (1 << 26) // channels))
        stream, branch = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        if op == "norm_fwd":
            return _norm_fwd(rows, channels, stream, branch, fmt, rng.random() < 0.8, pad)
        return _norm_bwd(rows, channels, stream, branch, fmt, rng.choice(["ck", "h"]), pad)
    if op.startswith("act"):
        act = rng.choice(["relu", "gelu", "silu", "swiglu"])
        channels = _log(rng, 16, 16384)
        channels = channels if rng.random() < 0.3 else max(16, channels // 32 * 32)
        channels += channels % 2 if act == "swiglu" else 0
        return _act(op, _log(rng, 1, min(1 << 17, (1 << 27) // channels)), channels, rng.choice(["f32", "bf16"]), fmt, act, pad)
    if op == "wgrad":
        cin, cout = (_log(rng, 16, 4096) for _ in range(2))
        if rng.random() < 0.6:
            cin, cout = max(16, cin // 32 * 32), max(16, cout // 32 * 32)
        dtype = rng.choice(["f32", "bf16", "bf16"])
        return _wgrad(_log(rng, 1, 16384 if dtype == "bf16" else 4096), cin, cout, dtype, fmt, rng.random() < 0.7, pad)
    vocab = _log(rng, 64, 131072)
    rows = _log(rng, 1, min(8192, (1 << 28) // vocab))
    return _logp(op, rows, vocab, rng.choice(["f32", "bf16"]), rng.choice([0, 1, 5, 20]) if op == "logp_fwd" else 0, rng.random() < 0.4, pad)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rand(g, rows, channels, dtype, pad=0, std=1.0):
    """Normal rows inside a buffer of rows pad elements longer."""
    buf = torch.empty(rows, channels + pad, dtype=DT[dtype], device="cuda")
    return buf.normal_(0.0, std, generator=g)[:, :channels]


def _like(rows, channels, dtype, pad=0):
    return torch.empty(rows, channels + pad, dtype=DT[dtype], device="cuda")[:, :channels]


def _activations(g, rows, channels, dtype, pad=0):
    """Activations of trained networks: channels of different spread, one in 64 several times the others."""
    x = _rand(g, rows, channels, dtype, pad)
    spread = torch.exp(0.3 * torch.randn(channels, device="cuda", generator=g))
    spread = torch.where(torch.rand(channels, device="cuda", generator=g) < 1 / 64, 5 * spread, spread)
    x.mul_(spread)
    return x


def _layout(rows, channels):
    pitch = -(-channels // GROUP) * GROUP
    at = -(-rows * pitch // 256) * 256
    groups, padded = -(-channels // 128), -(-rows // 64) * 64
    return pitch, at, groups, padded, at + groups * padded * 4


def _to_buffer(x, fmt):
    """The checkpoint of x: what an earlier forward pass has left in the user's buffer."""
    rows, channels = x.shape
    pitch, at, groups, padded, size = _layout(rows, channels)
    code, byte = _codes(x.float(), fmt)
    buf = torch.zeros(size, dtype=torch.uint8, device="cuda")
    buf[:rows * pitch] = (code.to(torch.int8) if fmt == "int8" else code.to(torch.float8_e4m3fn)).view(torch.uint8).reshape(-1)
    scales = buf[at:].view(groups, padded, 4)
    wide = torch.zeros(rows, groups * 4, dtype=torch.uint8, device="cuda")
    wide[:, :pitch // GROUP] = byte.to(torch.uint8)
    scales[:, :rows] = wide.view(rows, groups, 4).transpose(0, 1)
    return buf


def prepare(case, seed):
    c, g = case, _gen(seed)
    op, rows, pad = c["op"], c["rows"], c["pad"]
    s = {"case": case}
    if op.startswith("norm"):
        ch = c["channels"]
        gamma = 1 + 0.1 * torch.randn(ch, device="cuda", generator=g)
        x = _activations(g, rows, ch, c["stream"], pad)
        s |= dict(gamma=gamma)
        if op == "norm_fwd":
            s |= dict(x=x, r=_rand(g, rows, ch, c["branch"], pad, 0.3) if c["res"] else None,
                      h=_like(rows, ch, c["stream"], pad) if c["res"] else None, n=_like(rows, ch, c["branch"], pad),
                      rstd=torch.empty(rows, device="cuda"), ck=torch.empty(_layout(rows, ch)[-1], dtype=torch.uint8, device="cuda"),
                      kept=torch.empty(rows, ch, dtype=torch.bfloat16, device="cuda"))
        else:
            rstd = torch.rsqrt(x.float().square().mean(1) + EPS)
            s |= dict(dn=_rand(g, rows, ch, c["branch"], pad), dh=_rand(g, rows, ch, c["stream"], pad), dx=_like(rows, ch, c["stream"], pad),
                      dgamma=torch.empty(ch, device="cuda"), h=x if c["source"] == "h" else None,
                      ck=_to_buffer(x.float() * rstd[:, None], c["fmt"]) if c["source"] == "ck" else None, rstd=rstd if c["source"] == "ck" else None)
    elif op.startswith("act"):
        ch = c["channels"]
        out = ch // 2 if c["act"] == "swiglu" else ch
        x = _activations(g, rows, ch, c["dtype"], pad)
        if op == "act_fwd":
            s |= dict(x=x, a=_like(rows, out, c["dtype"], pad), ck=torch.empty(_layout(rows, ch)[-1], dtype=torch.uint8, device="cuda"),
                      kept=torch.empty(rows, ch, dtype=torch.bfloat16, device="cuda"))
        else:
            s |= dict(ck=_to_buffer(x, c["fmt"]), da=_rand(g, rows, out, c["dtype"], pad), dx=_like(rows, ch, c["dtype"], pad),
                      a_ck=torch.empty(_layout(rows, out)[-1], dtype=torch.uint8, device="cuda"),
                      kept=torch.empty(rows, out, dtype=torch.bfloat16, device="cuda"))
    elif op == "wgrad":
        x = _activations(g, rows, c["cin"], "f32")
        x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
        s |= dict(dy=_rand(g, rows, c["cout"], c["dtype"], pad), ck=_to_buffer(x, c["fmt"]),
                  gamma=1 + 0.1 * torch.randn(c["cin"], device="cuda", generator=g) if c["gamma"] else None,
                  dW=torch.empty(c["cout"], c["cin"], device="cuda"))
    else:
        v = c["vocab"]
        logits = _rand(g, rows, v, c["dtype"], pad, 2.5)
        live = v - v // 64 if c["masked"] else v
        logits[:, live:] = -math.inf                 # a vocabulary padded to a round size
        targets = torch.randint(0, live, (rows,), device="cuda", generator=g, dtype=torch.int32)
        targets = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.05, -1, targets)      # prompt and padding tokens
        s |= dict(logits=logits, targets=targets.to(torch.int32), lse=torch.empty(rows, device="cuda"), entropy=torch.empty(rows, device="cuda"))
        if op == "logp_fwd":
            s |= dict(logp=torch.empty(rows, device="cuda"), top_logp=torch.empty(rows, min(c["k"], v), device="cuda") if c["k"] else None,
                      top_index=torch.empty(rows, min(c["k"], v), device="cuda", dtype=torch.int32) if c["k"] else None)
        else:
            lse, ent = _stats(logits.float())[:2]
            s |= dict(lse=lse, entropy=ent, dlogp=torch.randn(rows, device="cuda", generator=g) - 1, dentropy=0.1 * torch.randn(rows, device="cuda", generator=g),
                      dlogits=_like(rows, v, c["dtype"], pad))
    return s


# ------------------------------------------------------------------ plain forms
def _codes(x, fmt):
    """x [rows][channels] float32 -> (code values [rows][pitch], scale bytes [rows][pitch / 32])."""
    rows, channels = x.shape
    x = torch.nn.functional.pad(x, (0, -channels % GROUP)).view(rows, -1, GROUP)
    amax = x.abs().amax(2)
    m, e = torch.frexp(amax)                         # amax = m 2^e, m in [1/2, 1)
    top_m, top_e = math.frexp(TOP[fmt])
    e = torch.where(amax > 0, torch.where(m <= top_m, e - top_e, e - top_e + 1), -117).clamp_min(-117)
    bad = ~torch.isfinite(amax)
    y = torch.ldexp(x, -e.unsqueeze(2))
    y = torch.round(y) if fmt == "int8" else y.to(torch.float8_e4m3fn).float()
    y = torch.where(bad.unsqueeze(2), 0.0, y)
    return y.view(rows, -1), torch.where(bad, 255, e + 127)


def _values(code, byte, channels):
    """What code values and scale bytes stand for, [rows][channels] float32."""
    y = code.view(code.shape[0], -1, GROUP) * torch.where(byte == 255, math.nan, torch.ldexp(torch.ones_like(byte, dtype=torch.float32), byte.int() - 127)).unsqueeze(2)
    return y.view(code.shape[0], -1)[:, :channels]


def _keep(x, fmt):
    return _values(*_codes(x, fmt), x.shape[1])


def _from_buffer(buf, rows, channels, fmt):
    pitch, at, groups, padded, size = _layout(rows, channels)
    code = buf[:rows * pitch].view(rows, pitch).view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()
    byte = buf[at:size].view(groups, padded, 4)[:, :rows].transpose(0, 1).reshape(rows, -1)[:, :pitch // GROUP]
    return _values(code, byte, channels)


def _activate(x, act):
    """-> (act(x), function from the gradient of that to the gradient of x)."""
    if act == "swiglu":
        gate, up = x.chunk(2, 1)
        sig = 1 / (1 + torch.exp(-gate))
        silu = gate * sig
        return silu * up, lambda da: torch.cat([da * up * sig * (1 + gate * (1 - sig)), da * silu], 1)
    if act == "relu":
        return torch.where(x > 0, x, 0.0), lambda da: torch.where(x > 0, da, 0.0)
    if act == "silu":
        sig = 1 / (1 + torch.exp(-x))
        return x * sig, lambda da: da * sig * (1 + x * (1 - sig))
    k = 2 * math.sqrt(2 / math.pi)                  # the tanh form of gelu: x / (1 + exp(-k (x + 0.044715 x^3)))
    sig = 1 / (1 + torch.exp(-k * (x + 0.044715 * x * x * x)))
    return x * sig, lambda da: da * (sig + x * sig * (1 - sig) * k * (1 + 3 * 0.044715 * x * x))


def _stats(x):
    """Rows of float32 logits -> (log of the sum of exponentials, entropy)."""
    m = x.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    d = x - m
    e = torch.exp(d)
    s = e.sum(1)
    t = torch.where(e > 0, d * e, 0.0).sum(1)
    return m[:, 0] + torch.log(s), torch.where(s > 0, torch.log(s) - t / s, 0.0)


def _top(x, k):
    """The k largest of each row, the lowest index first among equals: (values, indices)."""
    b = (x + 0.0).view(torch.int32)
    key = (b ^ ((b >> 31) & 0x7fffffff)).long() << 32
    key |= 0xffffffff - torch.arange(x.shape[1], device=x.device)
    index = 0xffffffff - (torch.topk(key, min(k, x.shape[1]), 1).values & 0xffffffff)
    return torch.gather(x, 1, index), index.to(torch.int32)


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "norm_fwd":
        h = s["x"].float()
        if s["r"] is not None:
            h = (h + s["r"].float()).to(DT[c["stream"]])
            stored, h = h, h.float()
        rstd = 1 / torch.sqrt(h.square().mean(1) + EPS)
        xh = h * rstd[:, None]
        out = dict(n=(xh * s["gamma"]).to(DT[c["branch"]]), rstd=rstd, kept=_keep(xh, c["fmt"]).bfloat16())
        return dict(out, h=stored) if s["r"] is not None else out
    if op == "norm_bwd":
        if s["h"] is not None:
            h = s["h"].float()
            rstd = 1 / torch.sqrt(h.square().mean(1) + EPS)
            xh = h * rstd[:, None]
        else:
            rstd, xh = s["rstd"], _from_buffer(s["ck"], c["rows"], c["channels"], c["fmt"])
        dn = s["dn"].float()
        gd = dn * s["gamma"]
        dx = s["dh"].float() + rstd[:, None] * (gd - xh * (gd * xh).mean(1, keepdim=True))
        return dict(dx=dx.to(DT[c["stream"]]), dgamma=(dn * xh).sum(0))
    if op == "act_fwd":
        x = s["x"].float()
        return dict(a=_activate(x, c["act"])[0].to(DT[c["dtype"]]), kept=_keep(x, c["fmt"]).bfloat16())
    if op == "act_bwd":
        a, back = _activate(_from_buffer(s["ck"], c["rows"], c["channels"], c["fmt"]), c["act"])
        return dict(dx=back(s["da"].float()).to(DT[c["dtype"]]), kept=_keep(a, c["fmt"]).bfloat16())
    if op == "wgrad":
        dW = s["dy"].float().T @ _from_buffer(s["ck"], c["rows"], c["cin"], c["fmt"])
        return dW * s["gamma"] if s["gamma"] is not None else dW
    x, targets = s["logits"].float(), s["targets"].long()
    if op == "logp_fwd":
        lse, ent = _stats(x)
        picked = torch.gather(x, 1, targets.clamp_min(0)[:, None])[:, 0] - lse
        out = dict(logp=torch.where(targets >= 0, picked, 0.0), entropy=ent, lse=lse)
        if c["k"]:
            value, index = _top(x, c["k"])
            out |= dict(top_logp=value - lse[:, None], top_index=index)
        return out
    logq = x - s["lse"][:, None]
    p = torch.exp(logq)
    dx = -p * torch.where(targets >= 0, s["dlogp"], 0.0)[:, None] - s["dentropy"][:, None] * torch.where(p > 0, p * (logq + s["entropy"][:, None]), 0.0)
    dx.scatter_add_(1, targets.clamp_min(0)[:, None], torch.where(targets >= 0, s["dlogp"], 0.0)[:, None])
    return dx.to(DT[c["dtype"]])


# ------------------------------------------------------------------ the library's operators
_ctx = None


def _context(B):
    """One library context per process, as a program keeps it."""
    global _ctx
    if _ctx is None:
        _ctx = B.Context(0)
    return _ctx


def _own(s):
    from paper_1707_04585_b200 import binding as B
    ctx, c = _context(B), s["case"]
    op, rows, pad = c["op"], c["rows"], c["pad"]
    if op.startswith("norm"):
        ch = c["channels"]
        d = B.norm_desc(rows, ch, c["stream"], c["branch"], EPS, c["fmt"], ld_stream=ch + pad, ld_branch=ch + pad)
        if op == "norm_fwd":
            B.revnet_rmsnorm_fwd(ctx, d, s["x"], s["r"], s["gamma"], s["h"], s["n"], s["ck"], s["rstd"])
            B.revnet_act_load(ctx, B.act_desc(rows, ch, "bf16", c["fmt"]), s["ck"], s["kept"])
            out = dict(n=s["n"], rstd=s["rstd"], kept=s["kept"])
            return dict(out, h=s["h"]) if s["r"] is not None else out
        if "ws" not in s:
            s["ws"] = torch.empty(B.revnet_rmsnorm_workspace_bytes(ctx, d), dtype=torch.uint8, device="cuda")
        B.revnet_rmsnorm_bwd(ctx, d, s["dn"], s["dh"], s["h"], s["ck"], s["rstd"], s["gamma"], s["dx"], None, s["dgamma"], s["ws"])
        return dict(dx=s["dx"], dgamma=s["dgamma"])
    if op.startswith("act"):
        ch = c["channels"]
        out = ch // 2 if c["act"] == "swiglu" else ch
        d = B.act_desc(rows, ch, c["dtype"], c["fmt"], c["act"], ld_x=ch + pad, ld_a=out + pad)
        if op == "act_fwd":
            B.revnet_act_store(ctx, d, s["x"], s["ck"], s["a"])
            B.revnet_act_load(ctx, B.act_desc(rows, ch, "bf16", c["fmt"]), s["ck"], s["kept"])
            return dict(a=s["a"], kept=s["kept"])
        B.revnet_act_bwd(ctx, d, s["ck"], s["da"], s["dx"], s["a_ck"])
        B.revnet_act_load(ctx, B.act_desc(rows, out, "bf16", c["fmt"]), s["a_ck"], s["kept"])
        return dict(dx=s["dx"], kept=s["kept"])
    if op == "wgrad":
        d = B.wgrad_desc(rows, c["cin"], c["cout"], c["dtype"], c["fmt"], ld_dy=c["cout"] + pad)
        if "ws" not in s:
            s["ws"] = torch.empty(B.revnet_linear_wgrad_workspace_bytes(ctx, d), dtype=torch.uint8, device="cuda")
        B.revnet_linear_wgrad(ctx, d, s["dy"], s["ck"], s["gamma"], s["dW"], s["ws"])
        return s["dW"]
    d = B.logprob_desc(rows, c["vocab"], c["dtype"], min(c["k"], c["vocab"]), ld=c["vocab"] + pad)
    if op == "logp_fwd":
        B.revnet_logprobs_fwd(ctx, d, s["logits"], s["targets"], s["logp"], s["entropy"], s["lse"], s["top_logp"], s["top_index"])
        out = dict(logp=s["logp"], entropy=s["entropy"], lse=s["lse"])
        return dict(out, top_logp=s["top_logp"], top_index=s["top_index"]) if c["k"] else out
    B.revnet_logprobs_bwd(ctx, d, s["logits"], s["targets"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], s["dlogits"])
    return s["dlogits"]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    op, rows = c["op"], c["rows"]
    if op.startswith("norm"):
        ch, sb, bb = c["channels"], BYTES[c["stream"]], BYTES[c["branch"]]
        if op == "norm_fwd":
            per = sb + bb + CK + (bb + sb if c["res"] else 0)
            return dict(bytes=rows * ch * per + 4 * rows + 4 * ch, flops=6 * rows * ch)
        per = bb + 2 * sb + (CK if c["source"] == "ck" else sb)
        return dict(bytes=rows * ch * per + (4 * rows if c["source"] == "ck" else 0) + 8 * ch, flops=10 * rows * ch)
    if op.startswith("act"):
        ch, b = c["channels"], BYTES[c["dtype"]]
        out = ch // 2 if c["act"] == "swiglu" else ch
        if op == "act_fwd":
            return dict(bytes=rows * (ch * (b + CK) + out * b), flops=10 * rows * ch)
        return dict(bytes=rows * (ch * (CK + b) + out * (b + CK)), flops=15 * rows * ch)
    if op == "wgrad":
        return dict(bytes=rows * c["cout"] * BYTES[c["dtype"]] + rows * c["cin"] * CK + 4 * c["cin"] * c["cout"], flops=2 * rows * c["cin"] * c["cout"])
    b, v = BYTES[c["dtype"]], c["vocab"]
    if op == "logp_fwd":
        return dict(bytes=rows * v * b + rows * (16 + 8 * min(c["k"], v)), flops=5 * rows * v)
    return dict(bytes=2 * rows * v * b + 20 * rows, flops=8 * rows * v)


# ------------------------------------------------------------------ the definitions in 64 bits
def _held(x, fmt):
    """The value that 8 bits with a shared power of two keep for each element of x (float64), from the definition of the format."""
    rows, channels = x.shape
    n = -(-channels // GROUP)
    y = torch.zeros(rows, n * GROUP, dtype=torch.float64, device=x.device)
    y[:, :channels] = x
    y = y.view(rows, n, GROUP)
    top = y.abs().max(dim=2, keepdim=True).values
    unit = torch.exp2(torch.round(torch.log2(torch.clamp(top / TOP[fmt], min=2.0 ** -117))))      # within a factor of two
    unit = torch.where(top > TOP[fmt] * unit, 2 * unit, unit)
    unit = torch.where((top <= TOP[fmt] * unit / 2) & (unit > 2.0 ** -117), unit / 2, unit)
    q = y / unit
    if fmt == "int8":
        q = torch.round(q)
    else:                                            # four significant bits, not below 2^-9
        step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(q.abs(), min=2.0 ** -40))), min=-6) - 3)
        q = torch.round(q / step) * step
    return (q * unit).view(rows, -1)[:, :channels]


def _read64(buf, rows, channels, fmt):
    """A checkpoint's values in float64, from its bytes."""
    pitch, at, groups, padded, size = _layout(rows, channels)
    raw = buf[:rows * pitch].view(rows, pitch)[:, :channels].to(torch.int64)
    if fmt == "int8":
        v = (raw - 256 * (raw > 127)).double()
    else:
        e, f = (raw >> 3) & 15, (raw & 7).double()
        v = torch.where(e > 0, (8 + f) * torch.exp2((e - 10).double()), f * 2.0 ** -9) * (1.0 - 2.0 * (raw >> 7).double())
    ch = torch.arange(channels, device=buf.device)
    scale = buf[at:size].view(groups, padded, 4)[ch // 128, :rows, ch % 128 // GROUP].T
    return v * torch.exp2(scale.double() - 127)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op, D = c["op"], torch.float64
    if op == "norm_fwd":
        h = s["x"].to(D)
        out = {}
        if s["r"] is not None:
            h = h + s["r"].to(D)
            out["h"] = h
            h = h.to(DT[c["stream"]]).to(D)          # the norm is of what is stored
        rms = (h.pow(2).sum(1, keepdim=True) / h.shape[1] + EPS).sqrt()
        return dict(out, n=h / rms * s["gamma"].to(D), rstd=1 / rms[:, 0], kept=_held(h / rms, c["fmt"]))
    if op == "norm_bwd":
        dn, dh, gamma = s["dn"].to(D), s["dh"].to(D), s["gamma"].to(D)
        if s["h"] is not None:
            h = s["h"].to(D)
            r = (h.pow(2).sum(1, keepdim=True) / h.shape[1] + EPS).pow(-0.5)
            xh = h * r
        else:
            r, xh = s["rstd"].to(D)[:, None], _read64(s["ck"], c["rows"], c["channels"], c["fmt"])
        along = torch.einsum("rc,rc,c->r", dn, xh, gamma) / xh.shape[1]
        return dict(dx=dh + r * (dn * gamma - along[:, None] * xh), dgamma=torch.einsum("rc,rc->c", dn, xh))
    if op.startswith("act"):
        x = (s["x"].to(D) if op == "act_fwd" else _read64(s["ck"], c["rows"], c["channels"], c["fmt"])).requires_grad_(op == "act_bwd")
        if c["act"] == "swiglu":
            half = x.shape[1] // 2
            a = x[:, :half] * torch.sigmoid(x[:, :half]) * x[:, half:]
        elif c["act"] == "relu":
            a = torch.clamp(x, min=0)
        elif c["act"] == "silu":
            a = x * torch.sigmoid(x)
        else:
            a = 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
        if op == "act_fwd":
            return dict(a=a, kept=_held(x, c["fmt"]))
        dx, = torch.autograd.grad(a, x, s["da"].to(D))
        return dict(dx=dx, kept=_held(a.detach(), c["fmt"]))
    if op == "wgrad":
        x = _read64(s["ck"], c["rows"], c["cin"], c["fmt"])
        return torch.einsum("to,tc->oc", s["dy"].to(D), x * s["gamma"].to(D) if s["gamma"] is not None else x)
    x, targets = s["logits"].to(D), s["targets"].long()
    if op == "logp_fwd":
        lse = torch.logsumexp(x, 1)
        logq = x - lse[:, None]
        out = dict(lse=lse, entropy=torch.special.entr(logq.exp()).sum(1), logp=torch.where(targets < 0, 0.0, logq.gather(1, targets.clamp_min(0)[:, None])[:, 0]))
        return dict(out, top_logp=logq.topk(min(c["k"], c["vocab"]), 1).values, top_index=None) if c["k"] else out
    q = torch.exp(x - s["lse"].to(D)[:, None])
    gp = torch.where(targets < 0, 0.0, s["dlogp"].to(D))[:, None]
    hot = torch.zeros_like(q).scatter_(1, targets.clamp_min(0)[:, None], 1.0)
    bent = torch.nan_to_num((x - s["lse"].to(D)[:, None] + s["entropy"].to(D)[:, None]) * q, nan=0.0)
    return gp * (hot - q) - s["dentropy"].to(D)[:, None] * bent
