"""The host side of the operators around the expert layer, without a GPU: refusals, which come before any HIP call, the
sizes that the host computes, and tensors of other devices."""
import ctypes
import inspect

import pytest

import test_expert_devices_cpu as stand
from paper_2608_00867_amd import nuna
from test_abi_cpu import no_gpu_only
from test_expert_cpu import INVALID, MISALIGNED, OVERLAP, P, UNSUPPORTED, refused
from test_expert_devices_cpu import BF16, E8M0, F8, F32, I32, Far, Library, Stand

torch = pytest.importorskip("torch")


@no_gpu_only
def test_norm_refuses():
    good = dict(x=P[0], xs=512, res=P[1], rs=512, w=P[2], wd=nuna.BF16, eps=1e-6, rows=64, cols=512, sum=P[3], ss=512, out=P[4], q=P[5],
                qs=P[6], kind=0, rstd=P[7], dtype=nuna.BF16, stream=None)
    refused("nuna_rms_norm", good, [
        (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(sum=None), INVALID), (dict(q=None), INVALID), (dict(qs=None), INVALID),
        (dict(out=None, q=None, qs=None), INVALID), (dict(res=None), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(dtype=nuna.F32), UNSUPPORTED),
        (dict(wd=5), UNSUPPORTED), (dict(kind=2), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
        (dict(eps=float("inf")), INVALID), (dict(cols=0), INVALID), (dict(cols=16385, xs=40000, rs=40000, ss=40000), UNSUPPORTED),
        (dict(rows=1 << 31), INVALID), (dict(xs=511), INVALID), (dict(rs=-1), INVALID), (dict(ss=100), INVALID), (dict(x=P[0] + 8), MISALIGNED),
        (dict(w=P[2] + 2), MISALIGNED), (dict(rstd=P[7] + 2), MISALIGNED), (dict(out=P[4] + 8), MISALIGNED), (dict(q=P[5] + 8), MISALIGNED),
        (dict(out=P[0]), OVERLAP), (dict(sum=P[0] + 1024), OVERLAP), (dict(sum=P[1], ss=520), OVERLAP), (dict(sum=P[0], ss=520), OVERLAP),
        (dict(out=P[3]), OVERLAP), (dict(q=P[4]), OVERLAP), (dict(rstd=P[6]), OVERLAP), (dict(sum=P[2]), OVERLAP),
        (dict(sum=P[1], x=P[1] + 64), OVERLAP)])
    for over in (dict(sum=P[1]), dict(sum=P[0]), dict(wd=nuna.F32), dict(rows=0, x=None, res=None, sum=None, out=None, q=None, qs=None)):
        assert nuna.lib().nuna_rms_norm(*{**good, **over}.values()) in (nuna.OK, nuna.ERR_HIP), nuna.last_error()


@no_gpu_only
def test_norm_grad_refuses():
    good = dict(dout=P[0], z=P[1], zs=512, w=P[2], wd=nuna.F32, rstd=P[3], dsum=P[4], rows=64, cols=512, dx=P[5], dw=P[6], ws=P[7],
                bytes=64 * 512 * 4, dtype=nuna.BF16, stream=None)
    refused("nuna_rms_norm_grad", good, [
        *((dict([(n, None)]), INVALID) for n in ("dout", "z", "w", "rstd", "dx", "dw", "ws")), (dict(bytes=64 * 512 * 4 - 1), INVALID),
        (dict(dtype=3), UNSUPPORTED), (dict(wd=2), UNSUPPORTED), (dict(zs=511), INVALID), (dict(cols=0), INVALID), (dict(rows=1 << 31), INVALID),
        (dict(dx=P[0]), OVERLAP), (dict(dx=P[1]), OVERLAP), (dict(dx=P[4] + 512), OVERLAP), (dict(dw=P[2]), OVERLAP), (dict(ws=P[5]), OVERLAP),
        (dict(dw=P[6] + 4), MISALIGNED), (dict(rstd=P[3] + 2), MISALIGNED)])
    assert nuna.lib().nuna_rms_norm_grad(*{**good, "dx": P[4]}.values()) in (nuna.OK, nuna.ERR_HIP)


def test_workspaces():
    assert nuna.rms_norm_grad_workspace(0, 100) == 0
    assert 0 < nuna.rms_norm_grad_workspace(10, 100) <= nuna.rms_norm_grad_workspace(1 << 30, 100) <= 1 << 20
    n = ctypes.c_size_t()
    L = nuna.lib()
    assert L.nuna_rms_norm_grad_workspace(4, 100, None) == INVALID
    assert L.nuna_rms_norm_grad_workspace(4, 40000, ctypes.byref(n)) == UNSUPPORTED
    assert nuna.expert_layer_few_workspace(0, 8, 128, 128) == 0 < nuna.expert_layer_few_workspace(64, 32, 65536, 65536) <= 1 << 30
    assert L.nuna_expert_layer_few_workspace(4, 8, 128, 128, None) == INVALID
    assert L.nuna_expert_layer_few_workspace(65, 8, 128, 128, ctypes.byref(n)) == UNSUPPORTED
    assert L.nuna_expert_layer_few_workspace(4, 33, 128, 128, ctypes.byref(n)) == UNSUPPORTED
    assert L.nuna_expert_layer_few_workspace(4, 8, 0, 128, ctypes.byref(n)) == INVALID


@no_gpu_only
def test_router_refuses():
    good = dict(z=P[0], stride=256, bias=P[1], T=64, E=256, k=8, score=1, norm=1, f=1.0, idx=P[2], w=P[3], dtype=nuna.F32, stream=None)
    common = [(dict(z=None), INVALID), (dict(T=-1), INVALID), (dict(T=1 << 30), INVALID), (dict(E=0), INVALID), (dict(E=1025, stride=1025), INVALID),
              (dict(k=0), INVALID), (dict(k=65), INVALID), (dict(E=4), INVALID), (dict(stride=255), INVALID), (dict(score=2), UNSUPPORTED),
              (dict(f=float("inf")), INVALID), (dict(f=float("nan")), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(z=P[0] + 4), MISALIGNED)]
    refused("nuna_route_topk", good, common + [
        (dict(idx=None), INVALID), (dict(w=None), INVALID), (dict(score=0), UNSUPPORTED), (dict(idx=P[0]), OVERLAP), (dict(w=P[2] + 4), OVERLAP),
        (dict(w=P[1]), OVERLAP), (dict(idx=P[2] + 2), MISALIGNED)])
    good = dict(g=P[0], z=P[1], stride=256, idx=P[2], T=64, E=256, k=8, score=0, norm=0, f=1.0, d=P[3], dtype=nuna.BF16, stream=None)
    refused("nuna_route_topk_grad", good, [c if "z" not in c[0] else (dict(z=c[0]["z"] and P[1] + 4), c[1]) for c in common] + [
        (dict(g=None), INVALID), (dict(idx=None), INVALID), (dict(d=None), INVALID), (dict(d=P[1]), OVERLAP), (dict(d=P[0]), OVERLAP),
        (dict(d=P[3] + 8), MISALIGNED)])


@no_gpu_only
def test_swiglu_refuses():
    good = dict(gu=P[0], off=P[1], groups=8, rows=64, inner=200, out=P[2], q=P[3], qs=P[4], kind=1, dtype=nuna.BF16, stream=None)
    common = [(dict(gu=None), INVALID), (dict(groups=0), INVALID), (dict(groups=1025), INVALID), (dict(rows=1 << 31), INVALID), (dict(inner=0), INVALID),
              (dict(inner=1 << 31), INVALID), (dict(out=None, q=None, qs=None), INVALID), (dict(q=None), INVALID), (dict(qs=None), INVALID),
              (dict(kind=2), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED), (dict(gu=P[0] + 8), MISALIGNED), (dict(q=P[3] + 4), MISALIGNED),
              (dict(off=P[1] + 2), MISALIGNED), (dict(out=P[0]), OVERLAP), (dict(q=P[2]), OVERLAP), (dict(qs=P[3] + 64), OVERLAP), (dict(qs=P[1]), OVERLAP)]
    refused("nuna_swiglu", good, common)
    refused("nuna_swiglu_grad", dict(dout=P[5], **good), common + [(dict(dout=None), INVALID), (dict(out=P[5]), OVERLAP), (dict(dout=P[5] + 2), MISALIGNED)])


@no_gpu_only
def test_few_refuses():
    Q = [P[7] + (i << 30) for i in range(1, 4)]
    good = dict(x=P[0], xs=512, idx=P[1], w=P[2], T=16, k=8, w1=P[3], s1=P[4], w2=P[5], s2=P[6], first=0, E=8, H=512, I=256, out=Q[0], ws=Q[1],
                bytes=nuna.expert_layer_few_workspace(16, 8, 512, 256), kind=0, dtype=nuna.BF16, stream=None)
    refused("nuna_expert_layer_few", good, [
        *((dict([(n, None)]), INVALID) for n in ("x", "idx", "w", "w1", "s1", "w2", "s2", "out", "ws")), (dict(T=65), UNSUPPORTED), (dict(T=-1), UNSUPPORTED),
        (dict(k=33), UNSUPPORTED), (dict(k=0), UNSUPPORTED), (dict(E=0), INVALID), (dict(E=1025), INVALID), (dict(H=0), INVALID), (dict(I=0), INVALID),
        (dict(H=65537, xs=65537), UNSUPPORTED), (dict(I=65537), UNSUPPORTED), (dict(xs=511), INVALID), (dict(bytes=good["bytes"] - 1), INVALID),
        (dict(kind=4), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(x=P[0] + 2), MISALIGNED), (dict(w1=P[3] + 8), MISALIGNED),
        (dict(ws=Q[1] + 4), MISALIGNED), (dict(w=P[2] + 2), MISALIGNED), (dict(out=P[0]), OVERLAP), (dict(out=P[3] + 1024), OVERLAP), (dict(ws=Q[0] + 512), OVERLAP),
        (dict(ws=P[1]), OVERLAP)])


# ------------------------------------------------------------------ tensors of other devices

T, K, E, H, N = 6, 2, 4, 256, 128
CALLS = {
    "rms_norm": dict(x=((T, H), BF16), weight=((H,), BF16), residual=((T, H), BF16), residual_out=((T, H), BF16), out=((T, H), BF16),
                     q_out=((T, H), F8), scale_out=((T, 4), E8M0), rstd=((T,), F32)),
    "rms_norm_grad": dict(dout=((T, H), BF16), z=((T, H), BF16), weight=((H,), F32), rstd=((T,), F32), dresidual=((T, H), BF16),
                          dx=((T, H), BF16), dweight=((H,), F32), workspace=((T * H * 4,), torch.uint8)),
    "route_topk": dict(logits=((T, E), F32), topk=K, score="sigmoid", bias=((E,), F32), topk_idx=((T, K), I32), weights=((T, K), F32)),
    "route_topk_grad": dict(dweights=((T, K), F32), logits=((T, E), F32), topk_idx=((T, K), I32), dlogits=((T, E), F32)),
    "swiglu": dict(gu=((T, 2 * N), BF16), offsets=((E + 1,), I32), out=((T, N), BF16), q_out=((T, N), F8), scale_out=((T, 4), F32)),
    "swiglu_grad": dict(dout=((T, N), BF16), gu=((T, 2 * N), BF16), offsets=((E + 1,), I32), out=((T, 2 * N), BF16), q_out=((T, 2 * N), F8),
                        scale_out=((T, 4), F32)),
    "expert_layer_few": dict(x=((T, H), BF16), topk_idx=((T, K), I32), weights=((T, K), F32), w1=((E, 2 * N, H), F8), w1_scale=((E, 2, 4), F32),
                             w2=((E, H, N), F8), w2_scale=((E, 2, 4), F32), out=((T, H), BF16), workspace=((T * K * 3 * N * 2,), torch.uint8)),
}
TENSORS = [(call, arg) for call, args in CALLS.items() for arg, v in args.items() if isinstance(v, tuple)]


def call(name, dev=0, **other):
    args = {k: Stand(*v, other.get(k, dev)) if isinstance(v, tuple) else v for k, v in CALLS[name].items()}
    return getattr(nuna, name)(**args, stream=7)


@pytest.fixture
def no_library(monkeypatch):
    nuna.rms_norm_grad_workspace(T, H)  # asked of the library itself, and kept
    nuna.expert_layer_few_workspace(T, K, H, N)
    monkeypatch.setattr(nuna, "lib", Library)
    monkeypatch.setattr(nuna, "_current_device", lambda: 0)


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_the_current_device_reach_the_library(no_library, name):
    with pytest.raises(Far):
        call(name)


@pytest.mark.parametrize("name,arg", TENSORS)
@pytest.mark.parametrize("dev", [1, -1])
def test_a_tensor_of_another_device_is_refused(no_library, name, arg, dev):
    with pytest.raises(ValueError):
        call(name, **{arg: dev})


@pytest.mark.parametrize("name", CALLS)
def test_another_device_than_the_current_one_is_refused(no_library, name):
    with pytest.raises(ValueError, match="current"):
        call(name, dev=1)


def test_every_tensor_is_listed():
    """Every argument of the calls that is no plain number or text is in CALLS."""
    plain = {"eps", "scale", "stream", "topk", "score", "normalize", "factor", "first_expert"}
    for name, args in CALLS.items():
        assert set(inspect.signature(getattr(nuna, name)).parameters) - plain <= set(args), name
    assert stand.CALLS.keys().isdisjoint(CALLS)
