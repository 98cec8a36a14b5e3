"""The expert layer on the GPU at the ends of its ranges: long rows, many groups, edges of the number formats.

Bounds as in test_moe_expert_gpu.py unless a test says otherwise.  This file comes after the tests that pin the map from
workgroups to XCDs, as that one does."""
import numpy as np
import pytest

import expert_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F8 = torch.float8_e4m3fn
E8M0 = torch.float8_e8m0fnu
ONE = 0x38  # 1.0 in e4m3


@pytest.fixture(scope="module")
def nuna():
    from paper_2608_00867_amd import nuna as n
    n.init()
    return n


def test_columns_past_2_to_29_of_fp32_results(nuna):
    """A row of results of more than 2^31 bytes: every column is where it belongs."""
    torch.cuda.empty_cache()
    k, width = (1 << 29) + 128, 128
    b = torch.zeros((k, width), dtype=torch.uint8, device="cuda")
    for x in (0, 5, (1 << 28) + 3, (1 << 29) - 1, 1 << 29, (1 << 29) + 77, k - 1):
        b[x, 0] = ONE + x % 7
    sb = torch.full((k, 4), 127, dtype=torch.uint8, device="cuda")
    a = torch.zeros((1, width), dtype=torch.uint8, device="cuda")
    a[0, 0] = ONE
    sa = torch.full((1, 4), 127, dtype=torch.uint8, device="cuda")
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    out = torch.full((1, 1, k), float("nan"), device="cuda")
    nuna.f8_wgrad(a.view(F8), sa.view(E8M0), b.view(F8), sb.view(E8M0), off, out)
    assert nuna.last_launch()["kernels"] == "k_f8_tiles_wgrad"
    assert bool((out[0, 0] == b[:, 0].contiguous().view(F8).float()).all())
    del b, sb, out
    torch.cuda.empty_cache()


def test_offsets_that_are_not_ascending_stay_in_the_buffers(nuna):
    """A wrong table may give wrong results, but nothing outside the outputs is written; here the group whose rows no other
    group names comes out right all the same."""
    rows, n, k = 300, 200, 256
    g = torch.Generator().manual_seed(1)
    a, sa = nuna.f8_quantize(torch.randn((rows, k), generator=g).cuda())
    b, sb = nuna.f8_quantize_blocks(torch.randn((6, n, k), generator=g).cuda())
    off = torch.tensor([250, 300, 0, 120, 40, 200, -7], dtype=torch.int32, device="cuda")
    whole = torch.full((rows * n + 512,), 7.0, device="cuda")
    out = whole[256:-256].view(rows, n)
    nuna.f8_matmul(a, sa, b, sb, out, offsets=off)
    assert bool((whole[:256] == 7).all()) and bool((whole[-256:] == 7).all())
    want = nuna.f8_matmul(a, sa, b[0], sb[0], out_dtype=torch.float32)
    assert bool((out[250:] - want[250:]).abs().max() < 1e-3 * want.abs().max())
    x = torch.randn((rows, 72), generator=g).cuda()
    raw = torch.full((72 * ref.cols_width(rows, 6) + 512,), 0x3C, dtype=torch.uint8, device="cuda")
    q = raw[256:-256].view(72, -1).view(F8)
    qc, sc = nuna.f8_quantize_cols(x, off, "f32", q)
    assert bool((raw[:256] == 0x3C).all()) and bool((raw[-256:] == 0x3C).all())
    whole = torch.full((6 * 72 * 72 + 512,), 7.0, device="cuda")
    nuna.f8_wgrad(qc, sc, qc, sc, off, whole[256:-256].view(6, 72, 72))
    assert bool((whole[:256] == 7).all()) and bool((whole[-256:] == 7).all())


def test_product_without_out_leaves_no_old_memory(nuna):
    """Rows that no group holds are zeros where the call makes the output itself, as moe_scatter_grad's are."""
    rows, n, k = 512, 1024, 256
    a, sa = nuna.f8_quantize(torch.randn((rows, k), device="cuda"))
    b, sb = nuna.f8_quantize_blocks(torch.randn((3, n, k), device="cuda"))
    off = torch.tensor([5, 100, 100, 300], dtype=torch.int32, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        for stream in (None, torch.cuda.Stream()):
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                old = torch.full((rows, n), float("nan"), dtype=dtype, device="cuda")
            torch.cuda.synchronize()
            del old
            out = nuna.f8_matmul(a, sa, b, sb, offsets=off, out_dtype=dtype, stream=stream)
            torch.cuda.synchronize()
            assert bool((out[:5] == 0).all()) and bool((out[300:] == 0).all()) and bool(out.isfinite().all())
            assert bool((out[5:300] != 0).any(1).all())
