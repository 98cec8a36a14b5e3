"""The expert layer's host side, without a GPU: refusals, in the order that they are documented in, and the sizes that the
host computes.  Every refusal comes before any HIP call, so made-up device pointers are never used."""
import ctypes

import pytest

import expert_ref as ref
from paper_2608_00867_amd import nuna
from test_abi_cpu import BASE, no_gpu_only

INVALID, UNSUPPORTED, MISALIGNED, OVERLAP = (nuna.ERR_INVALID_ARG, nuna.ERR_UNSUPPORTED, nuna.ERR_MISALIGNED,
                                             nuna.ERR_OVERLAP)
P = [BASE + (i << 34) for i in range(8)]  # eight buffers, far apart


def refused(fn, good, changes):
    """Each change of the good call's arguments gives its status and says why; the good call itself only lacks a device."""
    names = list(good)
    f = getattr(nuna.lib(), fn)
    assert f(*good.values()) in (nuna.OK, nuna.ERR_HIP), nuna.last_error()
    for change, want in changes:
        assert set(change) <= set(names), change
        st = f(*{**good, **change}.values())
        assert st == want, (change, st, nuna.last_error())
        assert nuna.last_error()


@no_gpu_only
def test_sort_refuses():
    good = dict(topk=P[0], T=64, k=8, first=0, experts=256, off=P[1], slot=P[2], row=P[3], ws=None, bytes=0, stream=None)
    refused("nuna_moe_sort", good, [
        (dict(topk=None), INVALID), (dict(off=None), INVALID), (dict(slot=None), INVALID), (dict(row=None), INVALID),
        (dict(T=-1), INVALID), (dict(T=1 << 28), INVALID), (dict(k=0), INVALID), (dict(k=1025), INVALID),
        (dict(experts=0), INVALID), (dict(experts=1025), INVALID),
        (dict(topk=P[0] + 2), MISALIGNED), (dict(row=P[3] + 1), MISALIGNED),
        (dict(slot=P[0] + 4), OVERLAP), (dict(row=P[2]), OVERLAP), (dict(off=P[2] + 64), OVERLAP),
        (dict(T=4000), INVALID), (dict(T=4000, ws=P[4], bytes=16), INVALID),
        (dict(T=4000, ws=P[0], bytes=1 << 20), OVERLAP)])


def test_sort_workspace():
    assert nuna.moe_sort_workspace(64, 8, 256) == 0
    most = nuna.moe_sort_workspace(1 << 27, 8, 1024)
    assert 0 < nuna.moe_sort_workspace(4000, 8, 256) <= most <= 4 << 20
    n = ctypes.c_size_t()
    assert nuna.lib().nuna_moe_sort_workspace(64, 8, 256, None) == INVALID
    assert nuna.lib().nuna_moe_sort_workspace(64, 8, 0, ctypes.byref(n)) == INVALID


@no_gpu_only
def test_gather_refuses():
    good = dict(x=P[0], stride=512, row=P[1], T=64, k=8, H=512, y=P[2], cap=512, dtype=nuna.BF16, stream=None)
    bad = [(dict(x=None), INVALID), (dict(row=None), INVALID), (dict(y=None), INVALID), (dict(dtype=2), UNSUPPORTED),
           (dict(stride=511), INVALID), (dict(stride=-1), INVALID), (dict(H=0), INVALID), (dict(H=(1 << 30) + 1), INVALID),
           (dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(cap=1 << 31), INVALID), (dict(x=P[0] + 8), MISALIGNED),
           (dict(y=P[2] + 2), MISALIGNED), (dict(row=P[1] + 2), MISALIGNED), (dict(y=P[0] + 64), OVERLAP),
           (dict(row=P[2]), OVERLAP)]
    refused("nuna_moe_gather", good, bad)
    good8 = dict(x=P[0], stride=512, row=P[1], T=64, k=8, H=512, y=P[2], scale=P[3], cap=512, dtype=nuna.BF16, kind=1,
                 stream=None)
    refused("nuna_moe_gather_f8", good8, bad + [(dict(scale=None), INVALID), (dict(kind=2), UNSUPPORTED),
                                                (dict(scale=P[2] + 16), OVERLAP), (dict(scale=P[3] + 4), MISALIGNED)])


@no_gpu_only
def test_scatter_refuses():
    good = dict(y=P[0], row=P[1], w=P[2], T=64, k=8, H=512, cap=512, out=P[3], dtype=nuna.BF16, stream=None)
    refused("nuna_moe_scatter", good, [
        (dict(y=None), INVALID), (dict(row=None), INVALID), (dict(out=None), INVALID), (dict(dtype=-1), UNSUPPORTED),
        (dict(H=0), INVALID), (dict(k=0), INVALID), (dict(cap=(1 << 30) + 1), INVALID), (dict(out=P[3] + 8), MISALIGNED),
        (dict(w=P[2] + 2), MISALIGNED), (dict(out=P[0] + 512), OVERLAP), (dict(w=P[3]), OVERLAP)])
    good = dict(dout=P[0], y=P[1], row=P[2], w=P[3], T=64, k=8, H=512, cap=512, dy=P[4], dw=P[5], dtype=nuna.F32,
                stream=None)
    refused("nuna_moe_scatter_grad", good, [
        (dict(dout=None), INVALID), (dict(y=None), INVALID), (dict(row=None), INVALID), (dict(w=None), INVALID),
        (dict(dy=None), INVALID), (dict(dw=None), INVALID), (dict(dtype=7), UNSUPPORTED), (dict(dy=P[1]), OVERLAP),
        (dict(dy=P[0] + 16), OVERLAP), (dict(dw=P[3]), OVERLAP), (dict(dw=P[4] + 4), OVERLAP), (dict(dw=P[5] + 1), MISALIGNED)])


@no_gpu_only
def test_quantisers_refuse():
    good = dict(x=P[0], stride=512, rows=64, cols=512, dtype=nuna.BF16, out=P[1], scale=P[2], kind=0, stream=None)
    common = [(dict(x=None), INVALID), (dict(out=None), INVALID), (dict(scale=None), INVALID), (dict(dtype=2), UNSUPPORTED),
              (dict(kind=-1), UNSUPPORTED), (dict(cols=0), INVALID), (dict(rows=1 << 31), INVALID),
              (dict(x=P[0] + 4), MISALIGNED), (dict(out=P[1] + 8), MISALIGNED), (dict(scale=P[2] + 4), MISALIGNED),
              (dict(out=P[0]), OVERLAP), (dict(scale=P[1] + 16), OVERLAP)]
    refused("nuna_f8_quantize", good, common + [(dict(stride=100), INVALID)])
    good = dict(x=P[0], batch=2, rows=64, cols=512, dtype=nuna.BF16, out=P[1], scale=P[2], kind=0, stream=None)
    refused("nuna_f8_quantize_blocks", good, common + [(dict(batch=-1), INVALID),
                                                       (dict(batch=1 << 30, rows=1 << 20), INVALID)])
    good = dict(x=P[0], stride=512, x_rows=64, slot=P[3], k=2, off=P[4], groups=8, rows=128, cols=512, dtype=nuna.BF16,
                out=P[1], scale=P[2], kind=0, stream=None)
    refused("nuna_f8_quantize_cols", good, common + [
        (dict(stride=100), INVALID), (dict(off=None), INVALID), (dict(groups=0), INVALID), (dict(groups=1025), INVALID),
        (dict(k=0), INVALID), (dict(slot=None), INVALID), (dict(x_rows=1 << 31), INVALID), (dict(slot=P[3] + 2), MISALIGNED),
        (dict(off=P[2]), OVERLAP)])


@no_gpu_only
def test_products_refuse():
    good = dict(a=P[0], sa=P[1], b=P[2], sb=P[3], off=P[4], groups=8, rows=64, n=512, k=512, out=P[5], kind=0,
                dtype=nuna.BF16, stream=None)
    common = [(dict(a=None), INVALID), (dict(sa=None), INVALID), (dict(b=None), INVALID), (dict(sb=None), INVALID),
              (dict(out=None), INVALID), (dict(off=None), INVALID), (dict(groups=0), INVALID), (dict(groups=1025), INVALID),
              (dict(n=0), INVALID), (dict(k=0), INVALID), (dict(rows=1 << 31), INVALID), (dict(kind=3), UNSUPPORTED),
              (dict(dtype=4), UNSUPPORTED), (dict(a=P[0] + 8), MISALIGNED), (dict(sb=P[3] + 4), MISALIGNED),
              (dict(out=P[5] + 2), MISALIGNED), (dict(off=P[4] + 2), MISALIGNED), (dict(out=P[2] + 64), OVERLAP),
              (dict(out=P[1]), OVERLAP)]
    refused("nuna_f8_matmul", good, common + [(dict(k=511), UNSUPPORTED), (dict(k=64), UNSUPPORTED)])
    refused("nuna_f8_wgrad", good, common)


@no_gpu_only
def test_products_refuse_rows_past_their_offsets():
    """Tiles of 256 rows are copied at 32-bit offsets: a row of 2^24 bytes or more would wrap."""
    most = (1 << 24) - 128
    far = [BASE + (i << 40) for i in range(6)]
    good = dict(a=far[0], sa=far[1], b=far[2], sb=far[3], off=None, groups=1, rows=300, n=300, k=most, out=far[5], kind=0,
                dtype=nuna.BF16, stream=None)
    refused("nuna_f8_matmul", good, [(dict(k=1 << 24), UNSUPPORTED), (dict(k=1 << 30), UNSUPPORTED)])
    good = dict(a=far[0], sa=far[1], b=far[2], sb=far[3], off=far[4], groups=8, rows=most - 8 * 128, n=300, k=300,
                out=far[5], kind=0, dtype=nuna.F32, stream=None)
    refused("nuna_f8_wgrad", good, [(dict(rows=most - 7 * 128), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED)])


@no_gpu_only
def test_nothing_to_do_needs_no_device():
    L = nuna.lib()
    assert L.nuna_moe_gather(None, 8, None, 0, 2, 8, None, 0, nuna.BF16, None) == nuna.OK
    assert L.nuna_moe_scatter(None, None, None, 0, 2, 8, 0, None, nuna.BF16, None) == nuna.OK
    assert L.nuna_f8_quantize(None, 8, 0, 8, nuna.BF16, None, None, 0, None) == nuna.OK
    assert L.nuna_f8_matmul(None, None, P[0], P[1], None, 1, 0, 16, 128, None, 0, nuna.BF16, None) == nuna.OK


def test_sizes_match_the_reference():
    for n in (1, 127, 128, 129, 511, 512, 513, 2880, 7168):
        assert nuna.f8_width(n) == ref.width(n) and nuna.f8_pitch(n) == ref.pitch(n)
        assert nuna.f8_cols_width(n, 5) == ref.cols_width(n, 5)


def test_columns_of_the_groups_do_not_meet():
    """128 * (offsets[g] / 128 + g) leaves every group's rows room of their own, inside the width."""
    import numpy as np
    g = np.random.default_rng(1)
    for _ in range(300):
        counts = g.integers(0, g.choice([2, 130, 700]), size=g.integers(1, 40))
        off = np.concatenate([[0], np.cumsum(counts)])
        start = off // 128 + np.arange(len(off))
        blocks = -(-counts // 128)
        assert (start[:-1] + blocks <= start[1:]).all()
        assert start[-1] * 128 <= ref.cols_width(int(off[-1]), len(counts))


def test_binding_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    cpu = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)  # noqa: E731
    table = cpu(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        nuna.moe_sort(table, 8)
    with pytest.raises(ValueError):
        nuna.moe_gather(cpu(4, 8), table, cpu(8, 8))
    with pytest.raises(ValueError):
        nuna.moe_scatter(cpu(8, 8), table)
    with pytest.raises(ValueError):
        nuna.f8_quantize(cpu(4, 8))
    with pytest.raises(ValueError):
        nuna.f8_quantize_blocks(cpu(4, 8))
    with pytest.raises(ValueError):
        nuna.f8_quantize_cols(cpu(4, 8), cpu(2, dtype=torch.int32))
