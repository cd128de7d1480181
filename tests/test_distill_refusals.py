"""What the loss on stored target logits and its gradient refuse before anything is launched (CPU: addresses are never read)."""
import pytest

from paper_2605_07230_b200 import binding as cb

K, V, N, H = 4, 100, 10, 8
AT = {name: 0x10000000 * (i + 1) for i, name in enumerate(("draft", "top", "ids", "lse", "feat", "seq", "loss", "saved", "total", "up", "grad"))}


def loss(**kw):
    a = dict(AT, dtype=cb.F32, stride=V, n=N, K=K, V=V, h=H, T=1.0, tau=0.5, c=2.0)
    a.update(kw)
    return cb.lib().cascade_distill_loss(a["draft"], a["dtype"], a["stride"], a["top"], a["ids"], a["n"], a["lse"], a["feat"], a["seq"],
                                         a["K"], a["V"], a["h"], a["T"], a["tau"], a["c"], a["loss"], a["saved"], a["total"], None)


def grad(**kw):
    a = dict(AT, dtype=cb.F32, stride=V, grad_stride=V, n=N, K=K, V=V, T=1.0, scale=1.0)
    a.update(kw)
    return cb.lib().cascade_distill_grad(a["draft"], a["dtype"], a["stride"], a["top"], a["ids"], a["n"], a["saved"], a["up"], a["scale"],
                                         a["K"], a["V"], a["T"], a["grad"], a["grad_stride"], None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw", [dict(draft=None), dict(top=None), dict(ids=None), dict(loss=None), dict(saved=None), dict(dtype=2), dict(dtype=-1),
                                dict(K=0), dict(V=0), dict(n=0), dict(h=0), dict(stride=V - 1), dict(stride=2**41), dict(T=0.0), dict(T=-1.0),
                                dict(T=NAN), dict(T=INF), dict(c=0.0), dict(c=NAN), dict(tau=NAN), dict(draft=AT["draft"] + 2),
                                dict(saved=AT["saved"] + 8), dict(loss=AT["loss"] + 1), dict(seq=AT["seq"] + 2), dict(total=AT["total"] + 2),
                                dict(loss=AT["draft"] + 4 * (K * V - 1)), dict(saved=AT["top"]), dict(total=AT["loss"] + 4 * (K - 1)),
                                dict(saved=AT["loss"]), dict(loss=AT["feat"] + 4 * K * H - 4), dict(total=AT["seq"]),
                                dict(loss=AT["lse"]),
                                # rows farther apart than 64 bits count: they meet what lies behind
                                dict(K=2**31 - 1, stride=2**40, total=None)])
def test_loss_refuses(kw):
    assert loss(**kw) == cb.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(draft=None), dict(top=None), dict(ids=None), dict(saved=None), dict(grad=None), dict(dtype=7), dict(K=0),
                                dict(V=0), dict(n=0), dict(stride=V - 1), dict(grad_stride=V - 1), dict(grad_stride=2**41), dict(T=0.0),
                                dict(T=NAN), dict(scale=NAN), dict(scale=INF), dict(grad=AT["grad"] + 1), dict(saved=AT["saved"] + 4),
                                dict(up=AT["up"] + 2), dict(grad=AT["draft"] + 4), dict(grad=AT["draft"], grad_stride=V + 1),
                                dict(grad=AT["top"]), dict(grad=AT["ids"] + 4), dict(grad=AT["saved"]), dict(grad=AT["up"])])
def test_gradient_refuses(kw):
    assert grad(**kw) == cb.ERR_INVALID_ARG


def test_sizes_past_32_bits():
    big = 2**31 - 65535
    for call in (loss, grad):
        extra = dict(grad_stride=big) if call is grad else {}
        assert call(V=big, stride=big, **extra) == cb.ERR_UNSUPPORTED_SHAPE
        assert call(n=big) == cb.ERR_UNSUPPORTED_SHAPE
