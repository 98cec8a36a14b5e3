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


# ------------------------------------------------------------------ helpers

def cut_rows(rows, groups, seed):
    """Offsets of `groups` groups of uneven sizes, some of them empty."""
    cuts = np.sort(np.random.default_rng(seed).integers(0, rows + 1, groups - 1))
    return np.concatenate([[0], cuts, [rows]]).astype(np.int32)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    t = t.detach().cpu()
    if t.dtype == E8M0:
        e = t.view(torch.uint8).numpy().astype(np.float64)
        return np.where(e == 255, np.nan, 2.0 ** (e - 127))
    if t.dtype == F8:
        return ref.E4M3[t.view(torch.uint8).numpy()]
    return t.double().numpy()


def values8(q, s, row_block=1):
    """Float64 values of an 8-bit matrix [n, k]."""
    blocks = q.shape[1] // 128
    return ref.dequantize(host(q), host(s)[:, :blocks], row_block)


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


EPS = 2.0 ** -24
RUN = 8  # consecutive values whose products the 8-bit instructions cut together


def sum_bound(a, b, k):
    """(k + 4) additions in fp32, each off by at most a unit in the last place, of a [r, k] by b [c, k]."""
    return 2 * (k + 4) * EPS * (np.abs(a) @ np.abs(b).T)


def cut_bound(a, b):
    """What the 8-bit instructions may lose besides: in every run of eight consecutive products, each of the seven others
    less than 2^-13 of the power of two at or below the largest."""
    p = np.abs(a[:, None, :] * b[None]).reshape(a.shape[0], b.shape[0], -1, RUN)
    return 7 * 2.0 ** -13 * p.max(3).sum(2)


def bounded(got, want, bound, what=""):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} out of bounds, first at {np.argwhere(bad)[0]}: " \
        f"{got[bad][0]} for {want[bad][0]}, bound {np.broadcast_to(bound, got.shape)[bad][0]}"


# ------------------------------------------------------------------ many groups

@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("groups,rows", [(65, 64), (128, 4000), (160, 700), (256, 5000), (1024, 2100)])
def test_products_of_many_groups(nuna, groups, rows, kind, out):
    n, k, off = 72, 128, cut_rows(rows, groups, groups)
    a, sa = nuna.f8_quantize(normal((rows, k), 1).cuda(), kind)
    b, sb = nuna.f8_quantize_blocks(normal((groups, n, k), 2).cuda(), kind)
    got = host(nuna.f8_matmul(a, sa, b, sb, offsets=dev(off), out_dtype=out))
    a64 = values8(a, sa)
    for g in np.flatnonzero(np.diff(off)):
        r = slice(off[g], off[g + 1])
        b64 = values8(b[g], sb[g], 128)
        want = a64[r] @ b64.T
        bound = sum_bound(a64[r], b64, k)
        if out == torch.bfloat16:
            bound = bound + 2.0 ** -8 * np.abs(want) + cut_bound(a64[r], b64)
        bounded(got[r], want, bound, f"group {g}")


@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("groups,rows", [(65, 64), (128, 4000), (160, 700), (256, 5000), (1024, 2100)])
def test_columns_and_gradient_of_many_groups(nuna, groups, rows, kind):
    n, k, off = 40, 24, cut_rows(rows, groups, groups + 1)
    dy, x = normal((rows, n), 3).bfloat16(), normal((rows, k), 4).bfloat16()
    (a, sa), (b, sb) = (nuna.f8_quantize_cols(t.cuda(), dev(off), kind) for t in (dy, x))
    for t, q, s in ((dy, a, sa), (x, b, sb)):
        want_q, want_s = ref.quantize(ref.columns(t.double().numpy(), off, rows), kind)
        assert np.array_equal(host(q), want_q) and np.array_equal(host(s)[:, :want_s.shape[1]], want_s)
    got = host(nuna.f8_wgrad(a, sa, b, sb, dev(off)))
    a64, b64 = values8(a, sa), values8(b, sb)
    for g in range(groups):
        at, c = 128 * (off[g] // 128 + g), off[g + 1] - off[g]
        u, v = a64[:, at:at + c], b64[:, at:at + c]
        bounded(got[g], u @ v.T, sum_bound(u, v, c), f"group {g}")


# ------------------------------------------------------------------ edges of the formats, strides, many choices

@pytest.mark.parametrize("kind", ["f32", "e8m0"])
def test_columns_of_bf16_at_the_edges(nuna, kind):
    """Infinities, NaN, zeros, subnormal and the smallest and largest magnitudes, along the columns of bf16 rows."""
    x = torch.zeros((256, 14))
    x[7, 0], x[130, 1], x[3, 2] = float("inf"), float("nan"), float("-inf")
    x[:, 3], x[:, 4] = 1e-38, 1e-40
    x[0, 5], x[200, 5] = 3.38e38, -3.38e38
    x[:, 6], x[:, 7] = 448, -0.0
    x[:128, 8], x[0, 8] = torch.linspace(0, 0.02, 128), 448
    x[:, 9] = 2.0 ** -120
    x[:, 10], x[:, 11] = normal((256,), 1) * 1e-38, normal((256,), 2) * 5e37
    x[0, 12], x[1, 12] = 1e-38, 2.0 ** -133
    x[:, 13] = 7
    x = x.bfloat16()
    with np.errstate(all="ignore"):
        want_q, want_s = ref.quantize(x.double().numpy().T, kind)
    q, s = nuna.f8_quantize_cols(x.cuda(), dev(np.array([0, 256], np.int32)), kind)
    assert np.array_equal(host(q)[:, :256], want_q, equal_nan=True)
    assert np.array_equal(host(s)[:, :2], want_s, equal_nan=True)
    rows_q, rows_s = nuna.f8_quantize(x.t().contiguous().cuda(), kind)
    assert torch.equal(rows_q.view(torch.uint8), q.view(torch.uint8)[:, :256])  # the sign of zero too
    assert np.isnan(want_s[0, 0]) and np.isnan(want_s[1, 1]) and np.isfinite(want_s[3:]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,extra", [(200, 3), (128, 8), (257, 31)])
def test_strided_rows_are_quantised_as_contiguous_ones(nuna, H, extra, dtype):
    rows, k, groups = 300, 2, 5
    x = normal((rows, H + extra), 1).to(dtype).cuda()[:, :H]
    assert not x.is_contiguous()
    off = dev(cut_rows(rows, groups, 2))
    for kind in ("f32", "e8m0"):
        for got, want in zip(nuna.f8_quantize_cols(x, off, kind), nuna.f8_quantize_cols(x.contiguous(), off, kind)):
            assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
        row_of = dev(np.random.default_rng(3).permutation(rows * k).astype(np.int32).reshape(rows, k))
        new = lambda: (torch.zeros((rows * k, ref.width(H)), dtype=torch.uint8, device="cuda").view(F8),  # noqa: E731
                       torch.zeros((rows * k, ref.pitch(H)), device="cuda").to(torch.float32 if kind == "f32" else E8M0))
        for got, want in zip(nuna.moe_gather(x, row_of, *new()), nuna.moe_gather(x.contiguous(), row_of, *new())):
            assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("k", [64, 65, 130, 1024])
def test_tokens_of_many_choices(nuna, k):
    """More choices than a wave has lanes, among them tokens whose choices of one span are all dropped."""
    T, H = 5, 264
    g = np.random.default_rng(k)
    row_of = g.permutation(T * k).astype(np.int32).reshape(T, k)
    row_of[g.random((T, k)) < 0.3] = -1
    row_of[1, :64] = -1
    row_of[2, 64:] = -1
    row_of[3] = -1
    x, y, w = normal((T, H), 1), normal((T * k, H), 2), normal((T, k), 3)
    here = row_of >= 0
    rows = row_of[here]
    out = nuna.moe_gather(x.cuda(), dev(row_of), torch.zeros((T * k, H), device="cuda"))
    want = np.zeros((T * k, H))
    want[rows] = np.repeat(x.double().numpy()[:, None], k, 1)[here]
    assert np.array_equal(host(out), want)
    y64, w64, d64 = y.double().numpy(), w.double().numpy(), x.double().numpy()
    terms = np.where(here[:, :, None], w64[:, :, None] * y64[np.maximum(row_of, 0)], 0)
    bounded(host(nuna.moe_scatter(y.cuda(), dev(row_of), w.cuda())), terms.sum(1), (k + 1) * EPS * np.abs(terms).sum(1))
    dy, dw = nuna.moe_scatter_grad(x.cuda(), y.cuda(), dev(row_of), w.cuda())
    want = np.zeros((T * k, H))
    want[rows] = (w64[:, :, None] * d64[:, None])[here]
    bounded(host(dy), want, 2.0 ** -23 * np.abs(want))
    each = np.where(here[:, :, None], y64[np.maximum(row_of, 0)] * d64[:, None], 0)
    bounded(host(dw), each.sum(2), (H + 1) * EPS * np.abs(each).sum(2))


# ------------------------------------------------------------------ what the sums hold

def outliers(rows, k, seed):
    """Rows with a few channels some 2^13 times the others, which cancel against weights of 1: what is left is the sum
    of the small ones, and a small one beside an outlier is the first thing that a sum of few bits loses."""
    g = np.random.default_rng(seed)
    a = g.choice([1, 1.125, 1.25, 1.5, 1.75, 1.875], (rows, k)) * 2.0 ** g.integers(-6, -4, (rows, 1))
    for r in range(rows):
        for block in range(0, k, 128):
            at = block + g.choice(128, 6, replace=False)
            a[r, at[:3]], a[r, at[3:]] = 256, -256
    return a


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("rows,n,k,kernel", [(3, 24, 128, "k_f8_few"), (20, 300, 512, "k_f8_few"),
                                             (300, 2101, 256, "k_f8_tiles"), (1000, 6201, 128, "k_f8_tiles")])
def test_blocks_with_outliers(nuna, rows, n, k, kernel, kind, out):
    """The values are held exactly in 8 bits with a scale of 1, so the error is the sum's alone.  Results in fp32 are held
    to fp32 sums, less than a tenth of what the 8-bit instructions may cut."""
    a = np.tile(outliers(min(rows, 40), k, rows), (-(-rows // 40), 1))[:rows]
    b = np.tile(2.0 ** np.arange(-1, 2)[:, None], (-(-n // 3), k))[:n]
    q = [torch.from_numpy(t).float().cuda().to(F8) for t in (a, b)]
    assert all(np.array_equal(host(t), w) for t, w in zip(q, (a, b)))

    def ones(r):
        s = torch.ones((r, ref.pitch(k)), device="cuda")
        return s if kind == "f32" else torch.full(s.shape, 127, dtype=torch.uint8, device="cuda").view(E8M0)

    got = host(nuna.f8_matmul(q[0], ones(rows), q[1], ones(-(-n // 128)), out_dtype=out))
    assert nuna.last_launch()["kernels"] == kernel
    few, cols = min(rows, 40), min(n, 3)  # the rest repeats these
    want, bound = a[:few] @ b[:cols].T, sum_bound(a[:few], b[:cols], k)
    if out == torch.bfloat16:
        cut = cut_bound(a[:few], b[:cols])
        assert (cut > 10 * bound).all()
        bound = bound + cut + 2.0 ** -8 * np.abs(want)
    spread = [np.tile(t, (-(-rows // few), -(-n // cols)))[:rows, :n] for t in (want, bound)]
    bounded(got, *spread)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("rows,n", [(2, 24), (300, 2101)])
def test_small_blocks_after_a_large_one(nuna, rows, n, kind, out):
    """The sum over the blocks is held in fp32: sums of 2^-19 of it and less are not lost from block to block."""
    k = 128 * 12
    a = np.zeros((rows, k))
    a[:, :128] = 256
    a[:, 128:-128:4] = 2.0 ** -4 * (1 + np.arange(rows)[:, None] % 3)
    a[:, -128:] = -256
    q = torch.from_numpy(a).float().cuda().to(F8), torch.ones((n, k), device="cuda").to(F8)

    def ones(r):
        s = torch.ones((r, ref.pitch(k)), device="cuda")
        return s if kind == "f32" else torch.full(s.shape, 127, dtype=torch.uint8, device="cuda").view(E8M0)

    got = host(nuna.f8_matmul(q[0], ones(rows), q[1], ones(-(-n // 128)), out_dtype=out))
    want = np.tile(a.sum(1)[:, None], (1, n))  # of numbers that fp32 holds exactly, bf16 with one rounding
    bounded(got, want, 2.0 ** -8 * np.abs(want) if out == torch.bfloat16 else 0)


# ------------------------------------------------------------------ which form runs

# (rows, n, k, groups): rows and columns of a tile and threads of a workgroup, of bf16 and of fp32 results.
FORMS = [((3, 30001, 256, 1), (16, 64, 256), None), ((13, 200, 640, 1), (16, 16, 512), None),
         ((29, 1001, 1200, 1), (16, 32, 512), None), ((200, 1021, 1300, 1), (32, 32, 512), None),
         ((300, 2101, 300, 1), (64, 64, 256), None), ((640, 4203, 384, 16), (64, 128, 256), None),
         ((1000, 6201, 384, 1), (128, 256, 512), None), ((2100, 6201, 600, 1), (256, 256, 512), (128, 256, 512)),
         ((2500, 5333, 384, 7), (256, 256, 512), (128, 256, 512))]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("size,tile,wide", FORMS)
def test_forms_of_the_product(nuna, size, tile, wide, kind, out):
    """The sizes that test_moe_expert_gpu.py checks the product at reach each of its forms: the launch has the workgroups
    that tiles of the named size need."""
    rows, n, k, groups = size
    by, bx, threads = wide if wide and out == torch.float32 else tile
    sd = torch.float32 if kind == "f32" else E8M0
    kp = ref.width(k)
    zeros = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda").view(F8)  # noqa: E731
    ones = lambda *s: torch.ones((*s, ref.pitch(k)), device="cuda").to(sd)  # noqa: E731
    off = dev(cut_rows(rows, groups, rows)) if groups > 1 else None
    lead = (groups,) if groups > 1 else ()
    nuna.f8_matmul(zeros(rows, kp), ones(rows), zeros(*lead, n, kp), ones(*lead, -(-n // 128)), offsets=off, out_dtype=out)
    ytiles = rows // by + min(groups, rows) if groups > 1 else -(-rows // by)
    launch = nuna.last_launch()
    assert (launch["grid"], launch["threads"]) == (-(-ytiles * -(-n // bx) // 8) * 8, threads)


@pytest.mark.parametrize("rows,groups", [(3300, 3), (600, 3)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
def test_forms_of_the_gradient(nuna, rows, groups, kind, out):
    n, k = 300, 513
    by, bx, threads = 128, 128, 256 if kind == "f32" and out == torch.float32 else 512
    off = dev(cut_rows(rows, groups, 1))
    a, b = (nuna.f8_quantize_cols(torch.zeros((rows, c), device="cuda"), off, kind) for c in (n, k))
    nuna.f8_wgrad(*a, *b, off, out_dtype=out)
    launch = nuna.last_launch()
    assert (launch["grid"], launch["threads"]) == (-(-groups * -(-n // by) * -(-k // bx) // 8) * 8, threads)


# ------------------------------------------------------------------ the ends of the range

@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("rows,n", [(3, 24), (300, 2101)])
def test_products_near_the_ends_of_the_range(nuna, rows, n, kind, out):
    """Blocks with values up to 3.1e38 beside small weights, and scales whose product is as small as 2^-118: results are
    what they should be, as every value and scale here is a power of two or a few of them."""
    k = 256
    x = torch.zeros((rows, k))
    x[0, :] = 2.0 ** 127          # scale 2^127 / 448, or 2^119
    x[1, :128], x[1, 128:] = 2.0 ** -60, 2.0 ** -61
    x[2:, ::16] = 1.75 * 2.0 ** 100
    a, sa = nuna.f8_quantize(x.cuda(), kind)
    b, sb = nuna.f8_quantize_blocks(torch.full((n, k), 2.0 ** -40).cuda(), kind)
    got = host(nuna.f8_matmul(a, sa, b, sb, out_dtype=out))
    a64, b64 = values8(a, sa), values8(b, sb, 128)
    want = np.tile((a64 @ b64[:1].T), (1, n))
    assert np.isfinite(want).all() and (want > 0).all()
    # 2^-24 for each of two scales, their product and the sum's steps; the values' products are all alike in a run.
    bounded(got, want, (2.0 ** -8 if out == torch.bfloat16 else 2 * (k + 4) * EPS) * want)


def test_fp32_results_of_values_past_bf16_are_infinite(nuna):
    """As nuna.h says: with power-of-two scales a value that quantising brings to 2^128 is infinite in fp32 results, and
    not in bf16 ones, whose scales meet in the product."""
    x = torch.zeros((2, 128))
    x[0, 3], x[1, 3] = 3.35e38, 3.1e38   # 256 and 240 times 2^120
    a, sa = nuna.f8_quantize(x.cuda(), "e8m0")
    b, sb = nuna.f8_quantize_blocks(torch.full((16, 128), 2.0 ** -10).cuda(), "e8m0")
    wide = nuna.f8_matmul(a, sa, b, sb, out_dtype=torch.float32)
    assert bool(torch.isinf(wide[0]).all()) and bool((wide[1] == 240 * 2.0 ** 110).all())
    assert bool((nuna.f8_matmul(a, sa, b, sb)[0].float() == 2.0 ** 118).all())
