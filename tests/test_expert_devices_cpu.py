"""The expert layer's binding refuses tensors of several devices, or of another device than the current one, before any
pointer reaches the library (CPU only: stand-ins for tensors of devices that need not be there)."""
import inspect

import pytest

from paper_2608_00867_amd import nuna

torch = pytest.importorskip("torch")

F8, E8M0, BF16, F32, I32 = (torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.bfloat16, torch.float32, torch.int32)


class Far(Exception):
    """Raised where a call would have reached the library."""


class Stand:
    """What the binding asks of a contiguous tensor."""

    def __init__(self, shape, dtype, dev=0):
        self.shape, self.dtype, self.dev = torch.Size(shape), dtype, dev
        self.is_cuda = dev >= 0
        self.device = f"device {dev}"

    def get_device(self):
        return self.dev

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def stride(self, i):
        return self.shape[i + 1:].numel()

    def data_ptr(self):
        return 1 << 20


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Far(name)
        return call


T, K, E, H, N = 6, 2, 4, 256, 128
TABLE, W = ((T, K), I32), ((T, K), F32)
CALLS = {
    "moe_sort": dict(topk_idx=TABLE, num_experts=E, offsets=((E + 1,), I32), slot_of=((T * K,), I32), row_of=TABLE),
    "moe_gather": dict(x=((T, H), BF16), row_of=TABLE, out=((T * K, H), BF16)),
    "moe_gather ": dict(x=((T, H), BF16), row_of=TABLE, out=((T * K, H), F8), scale_out=((T * K, 4), F32)),
    "moe_scatter": dict(y=((T * K, H), BF16), row_of=TABLE, weights=W, out=((T, H), BF16)),
    "moe_scatter_grad": dict(dout=((T, H), BF16), y=((T * K, H), BF16), row_of=TABLE, weights=W, dy=((T * K, H), BF16),
                             dweights=W),
    "f8_quantize": dict(x=((T, H), BF16), out=((T, H), F8), scale_out=((T, 4), F32)),
    "f8_quantize_blocks": dict(x=((T, H), BF16), out=((T, H), F8), scale_out=((1, 4), F32)),
    "f8_quantize_cols": dict(x=((T, H), BF16), offsets=((E + 1,), I32), out=((H, 512), F8), scale_out=((H, 4), F32),
                             slot_of=((T,), I32)),
    "f8_matmul": dict(a=((T, H), F8), a_scale=((T, 4), E8M0), b=((E, N, H), F8), b_scale=((E, 1, 4), E8M0),
                      out=((T, N), BF16), offsets=((E + 1,), I32)),
    "f8_wgrad": dict(a=((N, 512), F8), a_scale=((N, 4), F32), b=((H, 512), F8), b_scale=((H, 4), F32),
                     offsets=((E + 1,), I32), out=((E, N, H), F32)),
}
TENSORS = [(call, arg) for call, args in CALLS.items() for arg, v in args.items() if isinstance(v, tuple)]


def call(name, dev=0, **other):
    args = {k: Stand(*v, other.get(k, dev)) if isinstance(v, tuple) else v for k, v in CALLS[name].items()}
    return getattr(nuna, name.strip())(**args, stream=7)


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    nuna.moe_sort_workspace(T, K, E)  # asked of the library itself, and kept
    monkeypatch.setattr(nuna, "lib", Library)
    monkeypatch.setattr(nuna, "_current_device", lambda: 0, raising=False)


def test_every_operator_is_here():
    names = {n for n, f in inspect.getmembers(nuna, inspect.isfunction) if n.startswith(("moe_", "f8_"))}
    assert {c.strip() for c in CALLS} == names - {"moe_sort_workspace", "f8_width", "f8_pitch", "f8_cols_width"}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_the_current_device_reach_the_library(name):
    with pytest.raises(Far):
        call(name)


@pytest.mark.parametrize("name,arg", TENSORS)
@pytest.mark.parametrize("dev", [1, -1])
def test_a_tensor_of_another_device_is_refused(name, arg, dev):
    with pytest.raises(ValueError):
        call(name, **{arg: dev})


@pytest.mark.parametrize("name", CALLS)
def test_another_device_than_the_current_one_is_refused(name):
    with pytest.raises(ValueError, match="current"):
        call(name, dev=1)


def test_a_stream_of_another_device_is_refused():
    class Stream:
        cuda_stream, device_index = 7, 1

    with pytest.raises(ValueError, match="stream"):
        nuna.f8_quantize(Stand((T, H), BF16), out=Stand((T, H), F8), scale_out=Stand((T, 4), F32), stream=Stream())
