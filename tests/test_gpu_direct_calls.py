"""Calls that skip ctypes refuse what the checked ones refuse, at every entry point and for every tensor of it.  (Every wrong tensor here has at least the memory
that the call would touch.)"""
import pytest
import torch

from paper_1707_04585_b200 import binding as B
from tests import token_ref as ref

pytestmark = pytest.mark.gpu
ROWS, C, K = 6, 64, 3


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    B.revnet_check_device(c)
    c.close()


def rows(dtype=torch.float32, n=C):
    return torch.zeros(ROWS, n, dtype=dtype, device="cuda")


def flat(n, dtype=torch.float32):
    return torch.zeros(n, dtype=dtype, device="cuda")


def ck(n=C):
    return torch.zeros(ref.layout(ROWS, n)[4], dtype=torch.uint8, device="cuda")


def calls(ctx):
    """Entry point -> its descriptor and tensors by name, in the calls' order."""
    act, norm, wgrad, logp = B.act_desc(ROWS, C, "f32", act="silu"), B.norm_desc(ROWS, C, "f32", "bf16"), B.wgrad_desc(ROWS, C, C, "f32"), B.logprob_desc(ROWS, C, "f32", K)
    bf = torch.bfloat16
    nws, wws = (flat(n, torch.uint8) for n in (B.revnet_rmsnorm_workspace_bytes(ctx, norm), B.revnet_linear_wgrad_workspace_bytes(ctx, wgrad)))
    return {
        "act_store": (act, dict(x=rows(), ck=ck(), a=rows())),
        "act_load": (act, dict(ck=ck(), a=rows())),
        "act_bwd": (act, dict(ck=ck(), da=rows(), dx=rows(), a_ck=ck())),
        "rmsnorm_fwd": (norm, dict(x=rows(), r=rows(bf), gamma=flat(C), h=rows(), n=rows(bf), ck=ck(), rstd=flat(ROWS))),
        "rmsnorm_bwd": (norm, dict(dn=rows(bf), dh=rows(), h=rows(), ck=None, rstd=None, gamma=flat(C), dx=rows(), dr=rows(bf), dgamma=flat(C), workspace=nws)),
        "linear_wgrad": (wgrad, dict(dy=rows(), ck=ck(), gamma=flat(C), dW=flat(C * C), workspace=wws)),
        "logprobs_fwd": (logp, dict(logits=rows(), targets=flat(ROWS, torch.int32), logp=flat(ROWS), entropy=flat(ROWS), lse=flat(ROWS), top_logp=rows(n=K), top_index=rows(torch.int32, K))),
        "logprobs_bwd": (logp, dict(logits=rows(), targets=flat(ROWS, torch.int32), lse=flat(ROWS), entropy=flat(ROWS), dlogp=flat(ROWS), dentropy=flat(ROWS), dlogits=rows())),
    }


def wrong(name, t):
    """Tensors that must not be taken in the place of t."""
    yield "another device", t.cpu()
    yield "another shape", torch.cat([t, t])
    if name == "workspace":
        return                       # (any type will do, and the entry point looks at the size)
    if t.dtype == torch.uint8:
        yield "another type", t.view(torch.int8)
        yield "too small", t[:-1]
        yield "strided", torch.cat([t, t])[::2]
        return
    yield "another type", t.double() if t.is_floating_point() else t.long()
    if t.dim() == 2 and t.shape[1] == C:
        big = torch.cat([t, t], 1)
        yield "other row stride", big[:, :C]
        yield "transposed", torch.cat([t] * 12)[:C, :].t()[:ROWS]
        yield "strided channels", big[:, ::2]
    yield "strided", torch.cat([t, t], -1)[..., ::2]
    yield "sparse", t.to_sparse()


@pytest.mark.parametrize("entry", ["act_store", "act_load", "act_bwd", "rmsnorm_fwd", "rmsnorm_bwd", "linear_wgrad", "logprobs_fwd", "logprobs_bwd"])
def test_both_ways_refuse_the_same_tensors(ctx, entry, monkeypatch):
    desc, args = calls(ctx)[entry]
    direct, checked = getattr(B._direct, entry), getattr(B, "revnet_" + entry)
    assert direct(ctx.h.value, ctx.device, desc, *args.values()) == 0
    # the first tensor under another call's descriptor, one tensor more and one fewer, a handle that is none
    other = B.act_desc(ROWS, C) if entry.startswith("logp") else B.logprob_desc(ROWS, C)
    for bad in ((ctx.h.value, ctx.device, other, *args.values()), (ctx.h.value, ctx.device, desc, *args.values(), None), (ctx.h.value, ctx.device, desc, *list(args.values())[:-1]),
                (0, ctx.device, desc, *args.values()), (None, ctx.device, desc, *args.values()), (ctx.h.value, ctx.device + 1, desc, *args.values()), (ctx.h.value, -1, desc, *args.values())):
        assert direct(*bad) is None
    for name, t in args.items():
        if t is None:
            continue
        for what, bad in wrong(name, t):
            if what == "another shape" and (name == "workspace" or t.dtype == torch.uint8):
                continue             # (larger ones are fine)
            put = dict(args, **{name: bad})
            assert direct(ctx.h.value, ctx.device, desc, *put.values()) is None, (name, what)
            for skip in (False, True):
                with monkeypatch.context() as m:
                    if skip:
                        m.setattr(B, "_direct", None)
                    with pytest.raises((B.RevnetError, RuntimeError)):
                        checked(ctx, desc, *put.values())
    # what may be absent is absent in both ways
    optional = {"act_store": ["a"], "act_bwd": ["a_ck"], "rmsnorm_fwd": ["gamma", "n", "ck", "rstd"], "rmsnorm_bwd": ["dh", "gamma", "dr"], "linear_wgrad": ["gamma"],
                "logprobs_fwd": ["logp", "entropy", "lse"], "logprobs_bwd": ["dlogp", "dentropy"], "act_load": []}[entry]
    for name in optional:
        put = dict(args, **{name: None})
        assert direct(ctx.h.value, ctx.device, desc, *put.values()) == 0
        with monkeypatch.context() as m:
            m.setattr(B, "_direct", None)
            checked(ctx, desc, *put.values())
    torch.cuda.synchronize()


def test_other_threads_run_while_a_launch_waits_for_the_queue(ctx):
    """A stream takes so many launches ahead; the next one waits.  That must not hold up Python's other threads: a host function in front of it in the stream
    may need one."""
    import threading
    import time
    desc, args = calls(ctx)["act_load"]
    B.revnet_act_load(ctx, desc, *args.values())
    torch.cuda.synchronize()
    gaps, stop = [0.0], threading.Event()

    def beat():
        last = time.perf_counter()
        while not stop.is_set():
            time.sleep(0.001)
            now = time.perf_counter()
            gaps.append(now - last)
            last = now
    t = threading.Thread(target=beat)
    t.start()
    try:
        torch.cuda._sleep(2_500_000_000)             # clocks: more than a second of nothing
        begin = time.perf_counter()
        for _ in range(5000):
            B.revnet_act_load(ctx, desc, *args.values())
        waited = time.perf_counter() - begin
    finally:
        stop.set()
        t.join()
        torch.cuda.synchronize()
    assert waited > 0.5              # the launches did wait
    assert max(gaps) < 0.3
