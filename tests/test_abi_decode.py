"""What the decode entry points refuse, on any machine: the C ABI's status codes, which come before any device work, and the binding's checks."""
import ctypes

import pytest
import torch

from paper_2605_16360_amd import binding as pk

ONE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(18)      # never dereferenced: every call below fails its checks


@pytest.fixture()
def ctx():
    c = pk.proxykv_create(pk.make_config(1, 4, 2, 64, 1, 4, 128))
    yield c
    pk.proxykv_destroy(c)


ATTEND = dict(q=ONE, k=ONE, v=ONE, lens=ONE, dtype=pk.PROXYKV_BF16, rows=2, N=8, group=4, T=1, D=128, out=ONE, weight=ONE)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), "EINVAL"), (dict(k=None), "EINVAL"), (dict(v=None), "EINVAL"), (dict(out=None), "EINVAL"),
    (dict(rows=0), "EINVAL"), (dict(N=0), "EINVAL"), (dict(group=0), "EINVAL"), (dict(T=0), "EINVAL"), (dict(T=9), "EINVAL"), (dict(D=0), "EINVAL"),
    (dict(N=1 << 31), "EINVAL"), (dict(rows=1 << 21), "EINVAL"), (dict(rows=1 << 62, group=4), "EINVAL"), (dict(rows=-2, group=-4), "EINVAL"),
    (dict(q=ODD), "EINVAL"), (dict(k=ODD), "EINVAL"), (dict(v=ODD), "EINVAL"), (dict(out=ODD), "EINVAL"), (dict(lens=ODD), "EINVAL"), (dict(weight=ODD), "EINVAL"),
    (dict(dtype=7), "EINVAL"), (dict(dtype=pk.PROXYKV_FP32), "EUNSUPPORTED"), (dict(D=96), "EUNSUPPORTED"), (dict(D=256), "EUNSUPPORTED"),
    (dict(D=(1 << 32) + 128), "EUNSUPPORTED"),
])
def test_attend_refusals(ctx, change, status):
    a = {**ATTEND, **change}
    rc = pk.load().proxykv_attend(ctx.handle, a["q"], a["k"], a["v"], a["lens"], a["dtype"], a["rows"], a["N"], a["group"], a["T"], a["D"], a["out"],
                                  a["weight"], None)
    assert rc == getattr(pk, "PROXYKV_" + status)
    assert pk.load().proxykv_attend(None, *[ONE] * 4, 0, 2, 8, 4, 1, 128, ONE, ONE, None) == pk.PROXYKV_EINVAL


SHARED = dict(q=ONE, ks=ONE, vs=ONE, slens=ONE, k=ONE, v=ONE, lens=ONE, dtype=pk.PROXYKV_FP16, batch=2, heads=2, P=8, N=8, group=4, T=1, D=64,
              out=ONE, ws=ONE, w=ONE)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), "EINVAL"), (dict(ks=None), "EINVAL"), (dict(vs=None), "EINVAL"), (dict(out=None), "EINVAL"), (dict(k=None), "EINVAL"), (dict(v=None), "EINVAL"),
    (dict(batch=0), "EINVAL"), (dict(heads=0), "EINVAL"), (dict(P=0), "EINVAL"), (dict(N=-1), "EINVAL"), (dict(T=9), "EINVAL"), (dict(T=0), "EINVAL"),
    (dict(P=1 << 31), "EINVAL"), (dict(batch=1 << 20), "EINVAL"), (dict(ks=ODD), "EINVAL"), (dict(vs=ODD), "EINVAL"), (dict(slens=ODD), "EINVAL"),
    (dict(ws=ODD), "EINVAL"), (dict(dtype=pk.PROXYKV_FP32), "EUNSUPPORTED"), (dict(dtype=-1), "EINVAL"), (dict(D=80), "EUNSUPPORTED"),
])
def test_attend_shared_refusals(ctx, change, status):
    a = {**SHARED, **change}
    rc = pk.load().proxykv_attend_shared(ctx.handle, a["q"], a["ks"], a["vs"], a["slens"], a["k"], a["v"], a["lens"], a["dtype"], a["batch"], a["heads"],
                                         a["P"], a["N"], a["group"], a["T"], a["D"], a["out"], a["ws"], a["w"], None)
    assert rc == getattr(pk, "PROXYKV_" + status)


EVICT = dict(k=ONE, v=ONE, w=ONE, pos=ONE, lens=ONE, budgets=None, rows=2, N=8, budget=4, recent=2, D=128)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), "EINVAL"), (dict(v=None), "EINVAL"), (dict(w=None), "EINVAL"), (dict(lens=None), "EINVAL"),
    (dict(rows=0), "EINVAL"), (dict(rows=1 << 21), "EINVAL"), (dict(N=0), "EINVAL"), (dict(N=1 << 31), "EINVAL"), (dict(budget=0), "EINVAL"),
    (dict(budget=9), "EINVAL"), (dict(recent=-1), "EINVAL"), (dict(recent=5), "EINVAL"), (dict(budgets=ONE, recent=9), "EINVAL"), (dict(D=0), "EINVAL"),
    (dict(k=ODD), "EINVAL"), (dict(v=ODD), "EINVAL"), (dict(w=ODD), "EINVAL"), (dict(pos=ODD), "EINVAL"), (dict(lens=ODD), "EINVAL"),
    (dict(budgets=ODD), "EINVAL"), (dict(D=100), "EUNSUPPORTED"), (dict(D=512), "EUNSUPPORTED"),
])
def test_evict_refusals(ctx, change, status):
    a = {**EVICT, **change}
    rc = pk.load().proxykv_evict(ctx.handle, a["k"], a["v"], a["w"], a["pos"], a["lens"], a["budgets"], a["rows"], a["N"], a["budget"], a["recent"],
                                 a["D"], None)
    assert rc == getattr(pk, "PROXYKV_" + status)


def test_the_proxy_side_does_not_take_half_precision(ctx):
    lib = pk.load()
    assert lib.proxykv_score(ctx.handle, ONE, ONE, ONE, pk.PROXYKV_FP16, 8, 8, 4, ONE, None) == pk.PROXYKV_EINVAL
    assert lib.proxykv_score_self(ctx.handle, ONE, ONE, pk.PROXYKV_FP16, 8, ONE, None) == pk.PROXYKV_EINVAL


def test_the_binding_refuses_tensors_of_the_host(ctx):
    q, k = torch.zeros(2, 4, 1, 128, dtype=torch.bfloat16), torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be on the context's device"):
        pk.proxykv_attend(ctx, q, k, k)
    with pytest.raises(ValueError, match="q must be on"):
        pk.proxykv_attend_shared(ctx, q[None], k, k)
    with pytest.raises(ValueError, match="k must be on"):
        pk.proxykv_evict(ctx, k, k, torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), 4, 2)
    with pytest.raises(ValueError, match="go together"):
        pk.proxykv_attend_shared(ctx, q[None], k, k, k=k[None])
    with pytest.raises(ValueError, match="own tokens"):
        pk.proxykv_attend_shared(ctx, q[None], k, k, lens=torch.zeros(1, 2, dtype=torch.int32))
