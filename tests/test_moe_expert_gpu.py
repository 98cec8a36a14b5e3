"""The expert layer on the GPU against its definition in 64 bits (expert_ref): the slots sorted by expert, the rows
gathered, scattered and their gradients, the quantisers and the 8-bit products, at the sizes and masks where they can go
wrong.

Bounds.  Moves and integers are compared for equality, and quantised bytes and scales too: the rule fixes every rounding.
A sum of m fp32 terms is off by at most (m + 1) 2^-24 times the sum of its terms' magnitudes, a result rounded to bf16
by 2^-8 of itself besides.  The 8-bit matrix instructions cut each product of a block of 128 at 2^-13 of the largest,
which 2^-13 times the sum of the magnitudes covers.

These tests make streams of their own.  Where a process has used several, a launch's first workgroup need no longer run on
XCD 0, so the tests that pin the map from workgroups to XCDs come before this file."""
import numpy as np
import pytest

import expert_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 2.0 ** -24
CUT = 2.0 ** -13
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def nuna():
    from paper_2608_00867_amd import nuna as n
    n.init()
    return n


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    t = t.detach().cpu()
    if t.dtype == torch.float8_e8m0fnu:
        e = t.view(torch.uint8).numpy().astype(np.float64)
        return np.where(e == 255, np.nan, 2.0 ** (e - 127))
    if t.dtype == torch.float8_e4m3fn:
        return ref.E4M3[t.view(torch.uint8).numpy()]
    return t.double().numpy() if t.dtype.is_floating_point else t.numpy()


def values(shape, dtype, seed, spread=1.0):
    """N(0, 1) values whose columns differ in size, on the device, and the same in float64."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[-1:], generator=g))
    x = x.to(DTYPES[dtype])
    return x.cuda(), x.double().numpy()


def routing(T, k, E, seed, drop=0.0):
    g = np.random.default_rng(seed)
    t = np.argsort(g.random((T, E)), 1)[:, :k].astype(np.int32) if T else np.zeros((0, k), np.int32)
    return np.where(g.random(t.shape) < drop, -1, t).astype(np.int32)


def guarded(rows, cols, dtype, fill, pad=64):
    """A tensor between two bands of a bit pattern, and a check that the bands are whole."""
    whole = torch.empty(rows * cols + 2 * pad, dtype=dtype, device="cuda")
    raw = whole.view(torch.uint8)
    raw.fill_(0xA5)
    t = whole[pad:pad + rows * cols].view(rows, cols)
    t.view(torch.uint8).fill_(fill)

    def check():
        b = pad * whole.element_size()
        assert bool((raw[:b] == 0xA5).all()) and bool((raw[raw.numel() - b:] == 0xA5).all()), "write outside a buffer"
    return t, check


def bounded(got, want, bound, what=""):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} out of bounds, first at {np.argwhere(bad)[0]}: " \
        f"{got[bad][0]} for {want[bad][0]}, bound {np.broadcast_to(bound, got.shape)[bad][0]}"


# ------------------------------------------------------------------ sort

@pytest.mark.parametrize("T,k,E,first,count,drop", [
    (1, 1, 1, 0, 1, 0), (1, 8, 256, 0, 256, 0), (64, 8, 256, 32, 32, 0), (100, 3, 7, 2, 4, 0.3), (1024, 8, 1024, 0, 1024, 0),
    (1023, 8, 160, 0, 160, 0), (1025, 8, 64, 8, 8, 0.1), (4099, 8, 256, 0, 256, 0), (20011, 4, 33, 1, 31, 0.5),
    (70, 2, 1000, 999, 1, 0), (3000, 1, 2, 0, 2, 0), (333, 8, 16, 100, 5, 0)])
def test_sort(nuna, T, k, E, first, count, drop):
    topk = routing(T, k, E, T + E, drop)
    offsets, slot_of, row_of = ref.sort(topk, first, count)
    for _ in range(2):  # the same whatever the timing
        o, s, r = nuna.moe_sort(dev(topk), count, first)
        assert np.array_equal(host(o), offsets) and np.array_equal(host(s), slot_of) and np.array_equal(host(r), row_of)


def test_sort_takes_any_numbers(nuna):
    """Every int32 is a valid entry; the experts' range may end past int32's."""
    topk = np.array([[-2**31, 2**31 - 1, 5], [2**31 - 2, 0, -1], [5, 5, 5]], dtype=np.int32)
    for first, count in ((0, 6), (2**31 - 2, 10), (-2**31, 3), (4, 2)):
        for got, want in zip(nuna.moe_sort(dev(topk), count, first), ref.sort(topk, first, count)):
            assert np.array_equal(host(got), want), first


@pytest.mark.parametrize("T", [40, 3000])
def test_sort_one_expert_for_all_and_none(nuna, T):
    for e in (3, 9):
        topk = np.full((T, 8), e, dtype=np.int32)
        for got, want in zip(nuna.moe_sort(dev(topk), 8), ref.sort(topk, 0, 8)):
            assert np.array_equal(host(got), want)


def test_sort_nothing(nuna):
    o, s, r = nuna.moe_sort(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 5)
    assert o.tolist() == [0] * 6 and s.numel() == 0 and r.shape == (0, 4)


def test_sort_capped_grid_and_given_buffers(nuna):
    topk = routing(5000, 8, 64, 3)
    t = dev(topk)
    want = ref.sort(topk, 0, 64)
    ws = torch.full((nuna.moe_sort_workspace(5000, 8, 64),), 255, dtype=torch.uint8, device="cuda")
    bufs = [torch.full(w.shape, -7, dtype=torch.int32, device="cuda") for w in want]
    try:
        nuna.set_max_workgroups(3)
        got = nuna.moe_sort(t, 64, 0, *bufs, workspace=ws)
    finally:
        nuna.set_max_workgroups(0)
    assert nuna.last_launch()["grid"] <= 3
    assert all(g is b for g, b in zip(got, bufs)) and all(np.array_equal(host(g), w) for g, w in zip(got, want))


# ------------------------------------------------------------------ gather, scatter

ROWS = [(1, 1, 1, 8, 0), (1, 8, 16, 7168, 0), (7, 2, 8, 1, 0.4), (33, 4, 8, 100, 0.2), (64, 8, 32, 2880, 0), (300, 3, 4, 257, 0.5),
        (20, 12, 16, 129, 0), (513, 8, 64, 1024, 0.1), (9, 1, 3, 9000, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,E,H,drop", ROWS)
def test_gather(nuna, T, k, E, H, drop, dtype):
    topk = routing(T, k, E, T + H, drop)
    _, _, row_of = ref.sort(topk, 0, E)
    x, x64 = values((T, H), dtype, H)
    used = int((row_of >= 0).sum())
    for cap in {max(1, used), used + 5, max(1, used - 3)}:  # whole, room to spare, too small: rows past it are dropped
        out, check = guarded(cap, H, DTYPES[dtype], 0x3C)
        left = host(out[:1, :1])[0, 0]
        nuna.moe_gather(x, dev(row_of), out)
        want = np.full((cap, H), left)
        for t, j in np.argwhere((row_of >= 0) & (row_of < cap)):
            want[row_of[t, j]] = x64[t]
        assert np.array_equal(host(out), want)
        check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,extra", [(128, 3), (100, 28), (2048, 8)])
def test_gather_of_strided_rows(nuna, H, extra, dtype):
    T, k = 19, 2
    _, _, row_of = ref.sort(routing(T, k, 4, 1), 0, 4)
    wide, w64 = values((T, H + extra), dtype, 5)
    out = torch.zeros((T * k, H), dtype=DTYPES[dtype], device="cuda")
    nuna.moe_gather(wide[:, :H], dev(row_of), out)
    want = np.zeros((T * k, H))
    for t, j in np.argwhere(row_of >= 0):
        want[row_of[t, j]] = w64[t, :H]
    assert np.array_equal(host(out), want)
    q, s = nuna.f8_quantize(wide[:, :H])
    q2, s2 = nuna.f8_quantize(wide[:, :H].contiguous())
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s, s2)


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,E,H,drop", ROWS)
def test_scatter_and_its_gradient(nuna, T, k, E, H, drop, dtype, weighted):
    topk = routing(T, k, E, T + H, drop)
    _, _, row_of = ref.sort(topk, 0, E)
    cap = max(1, int((row_of >= 0).sum()) - 1)  # the last row is past the buffer
    here = (row_of >= 0) & (row_of < cap)
    y, y64 = values((cap, H), dtype, H + 1)
    g = np.random.default_rng(T)
    w = g.standard_normal((T, k)).astype(np.float32) if weighted else np.ones((T, k), np.float32)
    w[~here] = np.nan  # not read
    out, check = guarded(T, H, DTYPES[dtype], 0xFF)
    nuna.moe_scatter(y, dev(row_of), dev(w) if weighted else None, out)
    want, size = np.zeros((T, H)), np.zeros((T, H))
    for t, j in np.argwhere(here):
        want[t] += float(w[t, j]) * y64[row_of[t, j]]
        size[t] += abs(float(w[t, j])) * np.abs(y64[row_of[t, j]])
    bounded(host(out), want, (k + 1) * EPS * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0), "out")
    check()
    if not weighted:
        return
    dout, d64 = values((T, H), dtype, H + 2)
    dy, check = guarded(cap, H, DTYPES[dtype], 0x3C)
    left = host(dy[:1, :1])[0, 0]
    dw = torch.full((T, k), 7.0, device="cuda")
    nuna.moe_scatter_grad(dout, y, dev(row_of), dev(w), dy, dw)
    want_y, want_w, size_w = np.full((cap, H), left), np.zeros((T, k)), np.zeros((T, k))
    named = np.zeros((cap, 1), bool)
    for t, j in np.argwhere(here):
        r = row_of[t, j]
        want_y[r] = float(w[t, j]) * d64[t]
        named[r] = True
        want_w[t, j] = (d64[t] * y64[r]).sum()
        size_w[t, j] = np.abs(d64[t] * y64[r]).sum()
    rounding = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    bounded(host(dy), want_y, np.where(named, rounding * np.abs(want_y), 0), "dy")
    bounded(host(dw), want_w, (H + 1) * EPS * size_w, "dw")
    check()


def test_scatter_gradient_against_differences(nuna):
    """<dout, scatter(y + h u, w + h v) - scatter(y - h u, w - h v)> / 2h = <dy, u> + <dw, v>: exact for a product of two
    linear forms but for rounding."""
    T, k, E, H = 40, 4, 8, 192
    row_of = dev(ref.sort(routing(T, k, E, 1, 0.2), 0, E)[2])
    cap = T * k
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    y, w, dout, u, v, h = r(cap, H), r(T, k), r(T, H), r(cap, H), r(T, k), 2.0 ** -3
    dy, dw = nuna.moe_scatter_grad(dout, y, row_of, w)
    up = nuna.moe_scatter(y + h * u, row_of, w + h * v).double()
    down = nuna.moe_scatter(y - h * u, row_of, w - h * v).double()
    got = float((dy.double() * u.double()).sum() + (dw.double() * v.double()).sum())
    want = float((dout.double() * (up - down)).sum() / (2 * h))
    scale = float((dout.double().abs() * (up.abs() + down.abs())).sum() / (2 * h))
    assert abs(got - want) <= 64 * EPS * scale


def test_gather_and_scatter_are_adjoint(nuna):
    """<gather(x), z> = <x, scatter(z)> without weights: the gradient of the gather."""
    T, k, E, H = 50, 3, 8, 130
    row_of = dev(ref.sort(routing(T, k, E, 2, 0.3), 0, E)[2])
    g = torch.Generator(device="cuda").manual_seed(4)
    x, z = torch.randn((T, H), generator=g, device="cuda"), torch.randn((T * k, H), generator=g, device="cuda")
    y = nuna.moe_gather(x, row_of, torch.zeros((T * k, H), device="cuda"))
    back = nuna.moe_scatter(z, row_of)
    a, b = (y.double() * z.double()).sum(), (x.double() * back.double()).sum()
    assert abs(float(a - b)) <= 8 * EPS * float((y.double() * z.double()).abs().sum())


def test_scatter_spreads_what_is_not_finite_only_to_its_tokens(nuna):
    T, k, H = 6, 2, 64
    row_of = np.array([[0, 1], [2, -1], [-1, -1], [3, 4], [5, 99], [6, 7]], dtype=np.int32)
    y = torch.ones((8, H), device="cuda")
    y[1, 5], y[2, 6], y[7, 7] = float("nan"), float("inf"), float("-inf")
    out = host(nuna.moe_scatter(y, dev(row_of), torch.ones((T, k), device="cuda")))
    assert np.isnan(out[0, 5]) and out[1, 6] == np.inf and out[5, 7] == -np.inf
    assert np.isfinite(np.delete(out.reshape(-1), [5, H + 6, 5 * H + 7])).all()
    assert (out[2] == 0).all() and (out[4] == 1).all()


def test_rows_with_capped_grid(nuna):
    T, k, E, H = 100, 4, 8, 700
    row_of = dev(ref.sort(routing(T, k, E, 2), 0, E)[2])
    x, _ = values((T, H), "bf16", 1)
    y, _ = values((T * k, H), "bf16", 2)
    w = torch.rand((T, k), device="cuda")

    def all_of():
        out = nuna.moe_gather(x, row_of, torch.zeros((T * k, H), dtype=x.dtype, device="cuda"))
        q, s = nuna.moe_gather(x, row_of, torch.zeros((T * k, 768), dtype=torch.uint8, device="cuda").view(
            torch.float8_e4m3fn), torch.zeros((T * k, 8), device="cuda"))
        return [out, q.view(torch.uint8), s, nuna.moe_scatter(y, row_of, w), *nuna.moe_scatter_grad(x, y, row_of, w)]

    want = all_of()
    try:
        nuna.set_max_workgroups(5)
        got = all_of()
    finally:
        nuna.set_max_workgroups(0)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------ quantisers

def same_matrix(q, s, want_q, want_s, cols):
    got_s = host(s)
    n = ref.width(cols) // ref.BLOCK
    assert np.array_equal(got_s[..., :n], want_s, equal_nan=True)
    assert (got_s[..., n:] == 1).all()
    assert np.array_equal(host(q), want_q, equal_nan=True)


@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,k", [(1, 1), (1, 128), (3, 129), (5, 1000), (70, 2880), (2, 7168), (257, 512)])
def test_quantize_rows_and_blocks(nuna, n, k, dtype, kind):
    x, x64 = values((n, k), dtype, n + k, 2.0)
    q, check_q = guarded(n, ref.width(k), torch.uint8, 0x11)
    s, check_s = guarded(n, ref.pitch(k), torch.float32 if kind == "f32" else torch.uint8, 0x11)
    got = nuna.f8_quantize(x, kind, q.view(torch.float8_e4m3fn), s if kind == "f32" else s.view(torch.float8_e8m0fnu))
    same_matrix(*got, *ref.quantize(x64, kind), k)
    check_q()
    check_s()
    same_matrix(*nuna.f8_quantize_blocks(x, kind), *ref.quantize(x64, kind, 128), k)
    x3, x364 = values((3, n, k), dtype, n, 2.0)
    q3, s3 = nuna.f8_quantize_blocks(x3, kind)
    for i in range(3):
        same_matrix(q3[i], s3[i], *ref.quantize(x364[i], kind, 128), k)


@pytest.mark.parametrize("kind", ["f32", "e8m0"])
def test_quantize_edges(nuna, kind):
    """Zeros, the smallest and largest magnitudes, exact powers of two, what is not finite."""
    big = 3.0e38
    rows = np.zeros((12, 256), np.float32)
    rows[1, 3] = 1e-45
    rows[2, :] = 1e-38
    rows[3, 0], rows[3, 200] = big, -big
    rows[4, 7] = np.inf
    rows[5, 130] = np.nan
    rows[6, :] = 448
    rows[7, :] = np.nextafter(np.float32(448), np.float32(1000))
    rows[8, :128] = np.linspace(-1, 1, 128)
    rows[9, :] = -7.0
    rows[10, :] = 2.0 ** -120
    rows[11, 0], rows[11, 1:128] = 448, np.linspace(0, 0.02, 127)  # subnormal e4m3 values
    with np.errstate(all="ignore"):
        want_q, want_s = ref.quantize(rows.astype(np.float64), kind)
    q, s = nuna.f8_quantize(dev(rows), kind)
    same_matrix(q, s, want_q, want_s, 256)
    assert np.isnan(host(s)[4, 0]) and np.isfinite(host(s)[4, 1]) and np.isnan(host(q)[5, 128:]).all()
    # columns, by the same rule
    off = dev(np.array([0, 256], np.int32))
    qc, sc = nuna.f8_quantize_cols(dev(rows.T), off, kind)
    assert np.array_equal(host(qc)[:, :256], want_q, equal_nan=True)
    assert np.array_equal(host(sc)[:, :2], want_s, equal_nan=True)


@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,E,H,drop", ROWS)
def test_gather_quantised(nuna, T, k, E, H, drop, dtype, kind):
    topk = routing(T, k, E, T + H, drop)
    _, _, row_of = ref.sort(topk, 0, E)
    x, x64 = values((T, H), dtype, H)
    cap = max(1, int((row_of >= 0).sum()) - 1)
    q, check = guarded(cap, ref.width(H), torch.uint8, 0x3C)
    s = torch.full((cap, ref.pitch(H)), 3.0, device="cuda").to(torch.float32 if kind == "f32" else torch.uint8)
    s = s if kind == "f32" else s.view(torch.float8_e8m0fnu)
    untouched = host(s).copy()
    nuna.moe_gather(x, dev(row_of), q.view(torch.float8_e4m3fn), s)
    want_q, want_s = ref.quantize(x64, kind)
    got_q, got_s = host(q.view(torch.float8_e4m3fn)), host(s)
    named = np.zeros(cap, bool)
    for t, j in np.argwhere((row_of >= 0) & (row_of < cap)):
        r = row_of[t, j]
        named[r] = True
        assert np.array_equal(got_q[r], want_q[t]) and np.array_equal(got_s[r, :want_s.shape[1]], want_s[t])
        assert (got_s[r, want_s.shape[1]:] == 1).all()
    assert (q.cpu().numpy()[~named] == 0x3C).all() and np.array_equal(got_s[~named], untouched[~named])
    check()


GROUPS = [(1, [1]), (5, [5]), (0, [0, 0]), (300, [0, 300, 0]), (700, [128, 128, 1, 127, 256, 60]), (640, [640]),
          (1000, [3, 0, 0, 500, 129, 0, 368]), (50, [1] * 50)]


def offsets_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [1, 64, 200, 1025])
@pytest.mark.parametrize("rows,counts", GROUPS)
def test_quantize_cols(nuna, rows, counts, H, dtype, kind):
    off = offsets_of(counts)
    x, x64 = values((rows, H), dtype, H + rows, 1.0)
    width = ref.cols_width(rows, len(counts))
    q, check = guarded(H, width, torch.uint8, 0x3C)
    _, s = nuna.f8_quantize_cols(x, dev(off), kind, q.view(torch.float8_e4m3fn))
    same_matrix(q.view(torch.float8_e4m3fn), s, *ref.quantize(ref.columns(x64, off, rows), kind), width)
    check()


def test_quantize_cols_pulls_rows_through_slots(nuna):
    T, k, E, H = 90, 3, 5, 150
    topk = routing(T, k, E, 3, 0.2)
    off, slot_of, _ = ref.sort(topk, 0, E)
    x, x64 = values((T, H), "bf16", 9)
    rows = len(slot_of)
    pulled = np.zeros((rows, H))
    pulled[:off[-1]] = x64[slot_of[:off[-1]] // k]
    q, s = nuna.f8_quantize_cols(x, dev(off), "f32", slot_of=dev(slot_of), topk=k)
    same_matrix(q, s, *ref.quantize(ref.columns(pulled, off, rows), "f32"), ref.cols_width(rows, E))
    # A slot past x, or none, is a row of zeros.
    bad = slot_of.copy()
    bad[4], bad[5] = T * k + 7, -1
    pulled[4:6] = 0
    q, s = nuna.f8_quantize_cols(x, dev(off), "f32", slot_of=dev(bad), topk=k)
    same_matrix(q, s, *ref.quantize(ref.columns(pulled, off, rows), "f32"), ref.cols_width(rows, E))


# ------------------------------------------------------------------ products

def weights8(nuna, G, n, k, kind, seed):
    w, _ = values((G, n, k), "bf16", seed, 0.5)
    b, bs = nuna.f8_quantize_blocks(w, kind)
    kp = ref.width(k)
    s = host(bs)[:, :, :kp // 128]
    b64 = host(b) * np.repeat(np.repeat(s, 128, 1)[:, :n], 128, 2)
    return b, bs, b64


def rows8(nuna, rows, k, kind, seed):
    x, _ = values((rows, k), "bf16", seed)
    a, s = nuna.f8_quantize(x, kind)
    return a, s, ref.dequantize(host(a), host(s)[:, :ref.width(k) // 128])


def product_bound(want, size, k, out):
    if out == "bf16":
        return 2.0 ** -8 * np.abs(want) + (CUT + (k + 2) * EPS) * size
    return (k + 4) * EPS * size


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("rows,n,k", [(1, 1, 128), (1, 4096, 7168), (2, 16, 1), (3, 129, 256), (15, 40, 640), (16, 128, 1024),
                                      (17, 300, 384), (33, 1000, 2880), (64, 64, 128), (65, 257, 512), (130, 130, 896),
                                      (256, 384, 256), (300, 515, 1152), (777, 640, 384)])
def test_matmul(nuna, rows, n, k, kind, out):
    a, sa, a64 = rows8(nuna, rows, k, kind, rows + n)
    b, sb, b64 = weights8(nuna, 1, n, k, kind, n)
    o, check = guarded(rows, n, DTYPES[out], 0xFF)
    nuna.f8_matmul(a, sa, b[0], sb[0], o)
    want, size = a64 @ b64[0].T, np.abs(a64) @ np.abs(b64[0]).T
    bounded(host(o), want, product_bound(want, size, k, out), "out")
    check()


# One size for each form of the product: (rows, n, k, groups, the kernel).  Odd n, so that rows of out start anywhere and
# end inside 16 bytes; rows and blocks that end inside a tile.
FORMS = [(3, 30001, 256, 1, "k_f8_few"), (13, 200, 640, 1, "k_f8_few"), (29, 1001, 1200, 1, "k_f8_few"),
         (200, 1021, 1300, 1, "k_f8_few"), (300, 2101, 300, 1, "k_f8_tiles"), (640, 4203, 384, 16, "k_f8_tiles"),
         (1000, 6201, 384, 1, "k_f8_tiles"), (2100, 6201, 600, 1, "k_f8_tiles"), (2500, 5333, 384, 7, "k_f8_tiles")]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("rows,n,k,groups,kernel", FORMS)
def test_every_form_of_the_product(nuna, rows, n, k, groups, kernel, kind, out):
    cuts = np.sort(np.random.default_rng(rows).integers(0, rows + 1, groups - 1))
    off = np.concatenate([[0], cuts, [rows]]).astype(np.int32)
    a, sa, a64 = rows8(nuna, rows, k, kind, n)
    b, sb, b64 = weights8(nuna, groups, n, k, kind, rows)
    o, check = guarded(rows, n, DTYPES[out], 0xFF)
    if groups == 1:
        nuna.f8_matmul(a, sa, b[0], sb[0], o)
    else:
        nuna.f8_matmul(a, sa, b, sb, o, offsets=dev(off))
    assert nuna.last_launch()["kernels"] == kernel
    got = host(o)
    for g in range(groups):
        r = slice(off[g], off[g + 1])
        want, size = a64[r] @ b64[g].T, np.abs(a64[r]) @ np.abs(b64[g]).T
        bounded(got[r], want, product_bound(want, size, k, out), f"out of group {g}")
    check()


MANY = [(1, [1]), (4, [0, 3, 0, 1]), (40, [1] * 40), (70, [5, 0, 64, 1]), (200, [16, 17, 33, 100, 0, 34]), (520, [256, 1, 0, 263]),
        (600, [0, 0, 600]), (1300, [700, 90, 10, 500]), (0, [0, 0])]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("n,k", [(128, 256), (200, 384), (48, 1300)])
@pytest.mark.parametrize("rows,counts", MANY)
def test_matmul_grouped(nuna, rows, counts, n, k, kind, out):
    G, room = len(counts), 7
    off = offsets_of(counts)
    a, sa, a64 = rows8(nuna, rows + room, k, kind, rows + 1)
    b, sb, b64 = weights8(nuna, G, n, k, kind, n)
    o, check = guarded(rows + room, n, DTYPES[out], 0x3C)
    left = host(o[:1, :1])[0, 0]
    nuna.f8_matmul(a, sa, b, sb, o, offsets=dev(off))
    want, bound = np.full((rows + room, n), left), np.zeros((rows + room, n))
    for g in range(G):
        r = slice(off[g], off[g + 1])
        want[r] = a64[r] @ b64[g].T
        bound[r] = product_bound(want[r], np.abs(a64[r]) @ np.abs(b64[g]).T, k, out)
    bounded(host(o), want, bound, "out")
    check()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("n,k", [(128, 256), (72, 200), (300, 17)])
@pytest.mark.parametrize("rows,counts", MANY)
def test_wgrad(nuna, rows, counts, n, k, kind, out):
    G = len(counts)
    off = offsets_of(counts)
    x, _ = values((rows, k), "bf16", rows + 2)
    dy, _ = values((rows, n), "bf16", rows + 3)
    a, sa = nuna.f8_quantize_cols(dy, dev(off), kind)
    b, sb = nuna.f8_quantize_cols(x, dev(off), kind)
    blocks = a.shape[1] // 128
    a64, b64 = (ref.dequantize(host(q), host(s)[:, :blocks]) for q, s in ((a, sa), (b, sb)))
    o, check = guarded(G * n, k, DTYPES[out], 0xFF)
    nuna.f8_wgrad(a, sa, b, sb, dev(off), o.view(G, n, k))
    for g in range(G):
        at, c = 128 * (off[g] // 128 + g), counts[g]
        u, v = a64[:, at:at + c], b64[:, at:at + c]
        want = u @ v.T
        bounded(host(o.view(G, n, k)[g]), want, product_bound(want, np.abs(u) @ np.abs(v).T, c, out), f"group {g}")
    check()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("n,k", [(300, 203), (513, 130)])
def test_wgrad_of_many_rows(nuna, n, k, kind, out):
    """Groups of more than 1024 rows on average, one of them short."""
    test_wgrad(nuna, 3300, [2100, 7, 1193], n, k, kind, out)


def test_gradient_of_the_rows_is_the_product_with_the_transpose(nuna):
    """dx = dy W: the transposed weights' blocks have the same bytes and scales, so quantising before or after the
    transposition is the same."""
    rows, n, k = 37, 256, 384
    w, _ = values((n, k), "bf16", 5)
    q, s = nuna.f8_quantize_blocks(w)
    qt, st = nuna.f8_quantize_blocks(w.t().contiguous())
    assert torch.equal(q.view(torch.uint8).t(), qt.view(torch.uint8)) and torch.equal(s[:, :3].t(), st[:, :2])
    dy, sd, d64 = rows8(nuna, rows, n, "f32", 6)
    w64 = host(q) * np.repeat(np.repeat(host(s)[:, :3], 128, 0), 128, 1)
    got = nuna.f8_matmul(dy, sd, qt, st, out_dtype=torch.float32)
    want = d64 @ w64
    bounded(host(got), want, product_bound(want, np.abs(d64) @ np.abs(w64), n, "f32"))


def test_wgrad_against_differences(nuna):
    """<dy, (W + U) x - (W - U) x> = <dW, 2 U>.  The operands are integers up to 15 with power-of-two scales, which e4m3
    holds exactly, so what is left is the rounding of fp32 sums of integers."""
    rows, n, k, G = 90, 128, 128, 2
    off = dev(offsets_of([50, 40]))
    g = torch.Generator(device="cuda").manual_seed(7)
    small = lambda *s: torch.randint(-7, 8, s, generator=g, device="cuda").float()  # noqa: E731
    x, dy, w, u = small(rows, k), small(rows, n), small(G, n, k), small(G, n, k)
    a, sa = nuna.f8_quantize(x, "e8m0")
    y = []
    for weights in (w + u, w - u):
        b, sb = nuna.f8_quantize_blocks(weights, "e8m0")
        y.append(nuna.f8_matmul(a, sa, b, sb, offsets=off, out_dtype=torch.float32).double())
    dw = nuna.f8_wgrad(*nuna.f8_quantize_cols(dy, off, "e8m0"), *nuna.f8_quantize_cols(x, off, "e8m0"), off).double()
    want = float((dy.double() * (y[0] - y[1])).sum())
    got = float((dw * 2 * u.double()).sum())
    assert abs(got - want) <= 256 * EPS * float((dw.abs() * 2 * u.double().abs()).sum())


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
def test_products_keep_nan_in_its_rows(nuna, kind, out):
    rows, n, k = 40, 200, 512
    x, _ = values((rows, k), "bf16", 1)
    x[7, 300], x[8, 5] = float("nan"), float("inf")
    a, sa = nuna.f8_quantize(x, kind)
    b, sb, _ = weights8(nuna, 1, n, k, kind, 2)
    o = host(nuna.f8_matmul(a, sa, b[0], sb[0], out_dtype=DTYPES[out]))
    assert np.isnan(o[7:9]).all() and np.isfinite(np.delete(o, [7, 8], 0)).all()


def test_products_with_capped_grid(nuna):
    counts = [100, 3, 0, 200, 70]
    off, rows, n, k, G = dev(offsets_of(counts)), 373, 300, 384, 5
    a, sa, _ = rows8(nuna, rows, k, "f32", 1)
    b, sb, _ = weights8(nuna, G, n, k, "f32", 2)
    x, _ = values((rows, k), "bf16", 3)
    dy, _ = values((rows, n), "bf16", 4)

    def all_of():
        w = nuna.f8_quantize_blocks(x.view(1, rows, k))
        c1, c2 = nuna.f8_quantize_cols(dy, off), nuna.f8_quantize_cols(x, off)
        return [nuna.f8_matmul(a, sa, b, sb, offsets=off), nuna.f8_wgrad(*c1, *c2, off), w[0].view(torch.uint8), w[1],
                c1[0].view(torch.uint8), c1[1], nuna.f8_quantize(x)[1]]

    want = all_of()
    try:
        nuna.set_max_workgroups(3)
        got = all_of()
    finally:
        nuna.set_max_workgroups(0)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_offsets_outside_the_rows_are_cut(nuna):
    """Offsets that leave [0, rows] name no row outside the buffers."""
    rows, n, k = 50, 64, 128
    a, sa, a64 = rows8(nuna, rows, k, "f32", 1)
    b, sb, b64 = weights8(nuna, 3, n, k, "f32", 2)
    o, check = guarded(rows, n, torch.float32, 0)
    nuna.f8_matmul(a, sa, b, sb, o, offsets=dev(np.array([-5, 20, 30, 1000], np.int32)))
    want = np.concatenate([a64[r] @ b64[g].T for g, r in enumerate((slice(0, 20), slice(20, 30), slice(30, 50)))])
    bounded(host(o), want, product_bound(want, 1e3 + np.abs(want), k, "f32"))
    check()


# ------------------------------------------------------------------ streams, graphs, placement in memory

def layer(nuna, x, topk, weights, w1, s1, w2, s2, room):
    """One expert layer in serving form on the current stream."""
    E = w1.shape[0]
    offsets, _, row_of = nuna.moe_sort(topk, E)
    cap, kind = topk.numel(), s1.dtype
    xs = nuna.moe_gather(x, row_of, room["q1"], room["s1"])
    h = nuna.f8_matmul(*xs, w1, s1, room["h"], offsets=offsets)
    hq = nuna.f8_quantize(h, "f32" if kind == torch.float32 else "e8m0", room["q2"], room["s2"])
    y = nuna.f8_matmul(*hq, w2, s2, room["y"], offsets=offsets)
    assert cap == y.shape[0]
    return nuna.moe_scatter(y, row_of, weights, room["out"])


def layer_inputs(nuna, T, k, E, H, I, kind, seed):
    x, _ = values((T, H), "bf16", seed, 0.3)
    topk = dev(routing(T, k, E, seed))
    g = torch.Generator().manual_seed(seed)
    weights = torch.rand((T, k), generator=g).cuda()
    w1, s1 = nuna.f8_quantize_blocks(values((E, I, H), "bf16", seed + 1, 0)[0] * 0.1, kind)
    w2, s2 = nuna.f8_quantize_blocks(values((E, H, I), "bf16", seed + 2, 0)[0] * 0.1, kind)
    cap, sd = T * k, torch.float32 if kind == "f32" else torch.float8_e8m0fnu
    new8 = lambda n, c: torch.zeros((n, c), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
    room = dict(q1=new8(cap, ref.width(H)), s1=torch.zeros((cap, ref.pitch(H)), device="cuda").to(sd),
                h=torch.zeros((cap, I), dtype=torch.bfloat16, device="cuda"), q2=new8(cap, ref.width(I)),
                s2=torch.zeros((cap, ref.pitch(I)), device="cuda").to(sd),
                y=torch.zeros((cap, H), dtype=torch.bfloat16, device="cuda"),
                out=torch.zeros((T, H), dtype=torch.bfloat16, device="cuda"))
    return (x, topk, weights, w1, s1, w2, s2, room)


@pytest.mark.parametrize("T", [4, 1500])
def test_graph_replays_give_the_eager_result(nuna, T):
    """Captured once, replayed on new inputs with eager work between the replays."""
    args = layer_inputs(nuna, T, 4, 8, 256, 384, "f32", 1)
    layer(nuna, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(nuna, *args)
    for seed in (11, 12, 13):
        new = layer_inputs(nuna, T, 4, 8, 256, 384, "f32", seed)
        for old, fresh in zip(args[:3], new[:3]):
            old.copy_(fresh)
        args[-1]["out"].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = args[-1]["out"].clone()
        want = layer(nuna, *args).clone()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_other_streams(nuna):
    """Work enqueued on a given stream is ordered on it, and what is allocated for it belongs to it."""
    s = torch.cuda.Stream()
    x, _ = values((3000, 1024), "bf16", 1)
    topk = dev(routing(3000, 8, 64, 2))
    torch.cuda.synchronize()
    want = nuna.moe_sort(topk, 64)
    wq, ws = nuna.f8_quantize(x)
    torch.cuda.synchronize()
    for _ in range(3):
        got = nuna.moe_sort(topk, 64, stream=s)
        out = nuna.moe_gather(x, got[2], torch.zeros((24000, 1024), dtype=x.dtype, device="cuda"), stream=s)
        q, sc = nuna.f8_quantize(x, stream=s)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(q.view(torch.uint8), wq.view(torch.uint8)) and torch.equal(sc, ws)
        del got, out, q, sc


def test_offsets_past_32_bits(nuna):
    """Rows, bytes and weights past 2^31 elements."""
    H = 4096
    rows = (1 << 31) // H + 40
    y = torch.zeros((rows, H), dtype=torch.bfloat16, device="cuda")
    y[rows - 1] = 3.0
    y[rows - 2] = 5.0
    row_of = torch.tensor([[rows - 1, rows - 2], [0, rows - 1]], dtype=torch.int32, device="cuda")
    out = nuna.moe_scatter(y, row_of, torch.tensor([[1.0, 2.0], [1.0, 4.0]], device="cuda"))
    assert bool((out[0] == 13).all()) and bool((out[1] == 12).all())
    x = torch.full((2, H), 7.0, dtype=torch.bfloat16, device="cuda")
    nuna.moe_gather(x, row_of, y)
    assert bool((y[rows - 2:] == 7).all()) and bool((y[0] == 7).all()) and bool((y[1] == 0).all())
    del y
    # 3 groups of weights past 2^31 bytes in all: only the last has rows
    n, k = 1 << 15, 1 << 15
    b = torch.zeros((3, n, k), dtype=torch.uint8, device="cuda")
    b[2].fill_(0x38)  # 1.0
    sb = torch.ones((3, n // 128, k // 128), device="cuda")
    a = torch.full((3, k), 0x38, dtype=torch.uint8, device="cuda")
    sa = torch.full((3, k // 128), 0.5, device="cuda")
    f8 = torch.float8_e4m3fn
    got = nuna.f8_matmul(a.view(f8), sa, b.view(f8), sb, offsets=torch.tensor([0, 0, 0, 3], dtype=torch.int32, device="cuda"))
    assert bool((got == k / 2).all())


def test_launch_record(nuna):
    topk = dev(routing(64, 8, 256, 1))
    nuna.moe_sort(topk, 256)
    assert nuna.last_launch()["launches"] == 1
    nuna.moe_sort(dev(routing(4000, 8, 256, 1)), 256)
    assert nuna.last_launch()["launches"] == 2
