"""Expert products on the GPU against products in 64 bits, group by group.

Tolerances (u = 2^-24): a product of K terms accumulated in fp32, in whatever
order and grouping, is off by at most 2 K u of the sum of the terms' absolute
values; a bf16 result is rounded once more, 2^-8 of itself.
"""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(DT[dtype])


def _ends(counts):
    return torch.tensor(counts).cumsum(0).to(torch.int32).cuda()


def _bounds(counts):
    at = 0
    for e, c in enumerate(counts):
        yield e, at, at + c
        at += c


def _close(got, want, terms, K, dtype):
    bound = 2 * K * U * terms + 1e-38
    bound = bound + (2.0 ** -8 if dtype == "bf16" else U) * (want.abs() + bound)
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (int(bad.sum()), float(off.max()), float((off / bound).max()))


def _check_rows(x, w, counts, transposed, dtype, y):
    """y against x[i] @ w[e], zeros after the last group."""
    K = x.shape[1]
    want = torch.zeros(y.shape, dtype=torch.float64, device="cuda")
    terms = torch.zeros_like(want)
    for e, a, b in _bounds(counts):
        m = w[e].double().t() if transposed else w[e].double()
        want[a:b] = x[a:b].double() @ m
        terms[a:b] = x[a:b].double().abs() @ m.abs()
    _close(y, want, terms, K, dtype)


def _check_wgrad(x, dy, counts, out, dw):
    for e, a, b in _bounds(counts):
        want = x[a:b].double().t() @ dy[a:b].double()
        _close(dw[e], want, x[a:b].double().abs().t() @ dy[a:b].double().abs(), b - a, out)


# counts of each expert, k, n: single rows, tiles that end inside, empty experts at either end
# and between, more experts than a wave has lanes, sizes off every multiple
CASES = [
    ([1], 1, 1), ([1], 8, 8), ([0], 64, 64), ([3, 0, 2], 5, 7), ([0, 1, 0, 0, 1], 64, 128),
    ([17, 64, 1, 130], 96, 72), ([0, 65, 0, 63, 200, 0], 100, 136), ([256, 512], 64, 256),
    ([300, 1, 0, 255, 257], 200, 264), ([1] * 70 + [0] * 60 + [5] * 10, 72, 40), ([700], 515, 777),
    ([31, 33], 1000, 24), ([129, 127], 24, 1000), ([400, 0, 112], 768, 520), ([2, 3, 1, 2], 1024, 2048),
    ([9, 15, 0, 8, 40], 264, 520), ([1000, 24], 320, 384), ([513, 600], 576, 1032),
    # few tiles, a long summed index
    ([24, 9], 4096, 64), ([5, 0, 40], 3001, 50), ([6000], 64, 48), ([5000, 100, 3333], 33, 65),
    # many tiles
    ([900, 1200, 50, 0, 700], 1001, 1537), ([900, 1200, 50, 0, 700], 1024, 3200),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_products(case, dtype):
    counts, k, n = CASES[case]
    log(f"case: expert products {len(counts)} experts, {sum(counts)} rows, {k} x {n} {dtype}")
    g = torch.Generator(device="cuda")
    g.manual_seed(case)
    rows = sum(counts)
    x, dy = _randn(g, (rows, k), dtype), _randn(g, (rows, n), dtype)
    w = _randn(g, (len(counts), k, n), dtype)
    ends = _ends(counts)
    _check_rows(x, w, counts, False, dtype, tm.expert_matmul(x, w, ends))
    _check_rows(dy, w, counts, True, dtype, tm.expert_matmul(dy, w, ends, transposed=True))
    dw = tm.expert_wgrad(x, dy, ends)
    assert dw.dtype == torch.float32
    _check_wgrad(x, dy, counts, "f32", dw)
    if dtype == "bf16":
        _check_wgrad(x, dy, counts, "bf16", tm.expert_wgrad(x, dy, ends, dtype=torch.bfloat16))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_expert_are_zero(dtype):
    log("case: rows after the last expert's")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for counts, rows in (([100, 0, 60], 400), ([0, 0], 70), ([5, 3], 9)):
        x, dy = _randn(g, (rows, 128), dtype), _randn(g, (rows, 192), dtype)
        w = _randn(g, (len(counts), 128, 192), dtype)
        x[sum(counts):] = float("nan")   # whatever the padding holds
        dy[sum(counts):] = float("inf")
        y = tm.expert_matmul(x, w, _ends(counts))
        assert not y[sum(counts):].any()
        _check_rows(x, w, counts, False, dtype, y)
        _check_wgrad(x, dy, counts, "f32", tm.expert_wgrad(x, dy, _ends(counts)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k,n", [(128, 256), (200, 136), (75, 53)])
def test_nan_and_inf_stay_with_their_expert(k, n, dtype):
    """A neighbour's NaN must not reach a tile through rows that are loaded and not used."""
    log(f"case: NaN in one expert's rows and matrix {k} x {n} {dtype}")
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    counts = [70, 33, 130]
    x, dy = _randn(g, (233, k), dtype), _randn(g, (233, n), dtype)
    w = _randn(g, (3, k, n), dtype)
    ends = _ends(counts)
    ref = tm.expert_matmul(x, w, ends), tm.expert_matmul(dy, w, ends, transposed=True), tm.expert_wgrad(x, dy, ends)
    x[70:103] = float("nan")
    dy[70:103] = float("inf")
    w[1] = float("nan")
    got = tm.expert_matmul(x, w, ends), tm.expert_matmul(dy, w, ends, transposed=True), tm.expert_wgrad(x, dy, ends)
    for a, b in zip(ref[:2], got[:2]):
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[103:], b[103:]) and not b[70:103].isfinite().any()
    for e in (0, 2):
        assert torch.equal(ref[2][e], got[2][e])
    assert not got[2][1].isfinite().any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    log("case: expert products on strided operands")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    counts, k, n = [90, 0, 45, 200], 128, 192
    for pad in (64, 3):                       # 16-byte rows, and rows at any element
        xw = _randn(g, (335, k + pad), dtype)
        dyw = _randn(g, (335, n + pad), dtype)
        ww = _randn(g, (4, k + 2, n + pad), dtype)
        off = pad // 2
        x, dy, w = xw[:, off:off + k], dyw[:, off:off + n], ww[:, 1:k + 1, off:off + n]
        ends = _ends(counts)
        _check_rows(x, w, counts, False, dtype, tm.expert_matmul(x, w, ends))
        _check_rows(dy, w, counts, True, dtype, tm.expert_matmul(dy, w, ends, transposed=True))
        _check_wgrad(x, dy, counts, "f32", tm.expert_wgrad(x, dy, ends))
        turned = w.transpose(1, 2)            # columns contiguous: copied
        _check_rows(x, turned, counts, True, dtype, tm.expert_matmul(x, turned, ends, transposed=True))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_results_do_not_depend_on_what_else_is_in_the_call(dtype):
    """Bits of an expert's product: in a call of its own, and among others at another place."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    counts = [40, 100, 7]
    x, w = _randn(g, (147, 256), dtype), _randn(g, (3, 256, 128), dtype)
    y = tm.expert_matmul(x, w, _ends(counts))
    again = tm.expert_matmul(x, w, _ends(counts))
    assert torch.equal(y, again)
    for e, a, b in _bounds(counts):
        assert torch.equal(y[a:b], tm.expert_matmul(x[a:b].clone(), w[e:e + 1], _ends([b - a])))


def test_offsets_past_32_bits():
    """Rows and matrices whose element offsets pass 2^31."""
    log("case: expert products past 2^31 elements")
    rows, k, n = 40000, 65536, 24          # x: 2.6e9 elements, 5.2 GB
    x = torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x[-300:] = _randn(g, (300, k), "bf16")
    w = _randn(g, (2, k, n), "bf16", 0.1)
    ends = _ends([rows - 200, 200])
    y = tm.expert_matmul(x, w, ends)
    want = torch.cat([x[-300:-200].double() @ w[0].double(), x[-200:].double() @ w[1].double()])
    terms = torch.cat([x[-300:-200].double().abs() @ w[0].double().abs(), x[-200:].double().abs() @ w[1].double().abs()])
    _close(y[-300:], want, terms, k, "bf16")
    assert not y[:-300].any()
    dy = _randn(g, (rows, n), "bf16")
    dw = tm.expert_wgrad(x, dy, ends)
    for e, rng in ((0, slice(-300, -200)), (1, slice(-200, None))):
        _close(dw[e], x[rng].double().t() @ dy[rng].double(), x[rng].double().abs().t() @ dy[rng].double().abs(), rows, "f32")


def test_fp32_values_that_have_no_bf16_parts():
    """Values up to the largest fp32 and infinities take the fp32 products: the largest value
    times one stays, an infinity times a value is that infinity, not NaN; small and large
    entries in one product keep the accuracy of fp32."""
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    for rows, k, n in ((200, 96, 130), (700, 40, 1000)):
        x, w = _randn(g, (rows, k), "f32"), _randn(g, (1, k, n), "f32")
        x[3] = 0.0
        x[3, 5] = torch.finfo(torch.float32).max
        w[0, 5] = 1.0
        w[0, 7] = 0.5 + w[0, 7].abs()
        x[100, 7] = float("inf")
        y = tm.expert_matmul(x, w, _ends([rows]))
        assert (y[3] == torch.finfo(torch.float32).max).all()
        assert (y[100] == float("inf")).all()
        keep = torch.ones(rows, dtype=torch.bool, device="cuda")
        keep[3] = keep[100] = False
        want = x[keep].double() @ w[0].double()
        _close(y[keep], want, x[keep].double().abs() @ w[0].double().abs(), k, "f32")
        x = _randn(g, (rows, k), "f32") * torch.logspace(-20, 10, k, device="cuda")
        w = w * torch.logspace(15, -10, k, device="cuda")[None, :, None]
        want, terms = x.double() @ w[0].double(), x.double().abs() @ w[0].double().abs()
        _close(tm.expert_matmul(x, w, _ends([rows])), want, terms, k, "f32")
        dy = _randn(g, (rows, n), "f32", 1e-25)
        _check_wgrad(x, dy, [rows], "f32", tm.expert_wgrad(x, dy, _ends([rows])))


def test_ends_that_make_no_sense_stay_in_bounds():
    """Decreasing or too large ends: the rows that they reach are computed, nothing else is touched."""
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    x, w = _randn(g, (100, 64), "bf16"), _randn(g, (3, 64, 64), "bf16")
    guard = torch.full((300, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    for ends in ([50, 20, 1000], [-5, 100, 90], [2 ** 31 - 1, -2 ** 31, 5]):
        e = torch.tensor(ends, dtype=torch.int32, device="cuda")
        guard.fill_(7.0)
        out = guard[100:200]
        assert tm.lib().tm_expert_matmul(x.data_ptr(), 64, w.data_ptr(), 64, 4096, e.data_ptr(), out.data_ptr(), 64,
                                         100, 3, 64, 64, 0, 0, s) == 0
        assert (guard[:100] == 7).all() and (guard[200:] == 7).all()
        tm.expert_wgrad(x, x, e)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,k,n", [
    ([0, 7000, 1, 0, 513, 30, 0], 65, 33), ([1024, 1024, 0, 2048], 64, 72),
    # few tiles, groups of 256 rows and more on average
    ([3000, 40, 900, 0, 513, 30, 200, 1, 260, 700], 70, 65),
    # more experts than a wave has lanes, rows of none at the end
    ([3000 if e % 9 == 4 else 1200 * (e % 3) for e in range(70)], 8, 9),
])
def test_long_groups_in_chunks(counts, k, n, dtype):
    log(f"case: weight gradient of long uneven groups, {len(counts)} experts {k} x {n} {dtype}")
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    rows = sum(counts) + 700
    x, dy = _randn(g, (rows, k), dtype), _randn(g, (rows, n), dtype)
    x[rows - 700:] = float("nan")
    ends = _ends(counts)
    dw = tm.expert_wgrad(x, dy, ends)
    _check_wgrad(x, dy, counts, "f32", dw)
    assert torch.equal(dw, tm.expert_wgrad(x, dy, ends))
    for e, (c, m) in enumerate(zip(counts, dw)):
        assert c > 0 or not m.any(), e
    if dtype == "bf16":
        _check_wgrad(x, dy, counts, "bf16", tm.expert_wgrad(x, dy, ends, dtype=torch.bfloat16))


@pytest.mark.parametrize("counts,k,n", [([9, 3, 14], 7770, 461), ([100, 130], 6000, 700), ([7000], 900, 1400)])
def test_long_fp32_sums_keep_their_digits(counts, k, n):
    """Rounding errors of a sum of K terms in turn grow with sqrt(K): each rounding of the running sum is off by
    0.41 U of it (rms: evenly within half a unit in the last place, which is U to 2 U of the value), together
    0.41 U sqrt(K / 2) of the result.  Runs of less than a half of K stay below 0.29 of U sqrt(K / 2)."""
    log(f"case: long fp32 sums, {sum(counts)} rows, {k} x {n}")
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    rows, ends = sum(counts), _ends(counts)
    x, dy, w = _randn(g, (rows, k), "f32"), _randn(g, (rows, n), "f32"), _randn(g, (len(counts), k, n), "f32")
    if len(counts) > 1:
        got, K = tm.expert_matmul(x, w, ends), k
        want = torch.cat([x[a:b].double() @ w[e].double() for e, a, b in _bounds(counts)])
    else:
        got, K = tm.expert_wgrad(x, dy, ends)[0], rows
        want = x.double().t() @ dy.double()
    assert float((got.double() - want).norm()) <= 0.3 * U * (K / 2) ** 0.5 * float(want.norm())


def test_ends_that_make_no_sense_stay_in_bounds_of_the_chunks():
    """Decreasing ends count rows more than once: more chunks than the call has room for are left out."""
    log("case: weight gradient in chunks, ends that decrease")
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    rows = 4096
    x = _randn(g, (rows, 64), "bf16")
    for ends in ([rows, 0, rows], [-5, rows, 90], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]):
        dw = tm.expert_wgrad(x, x, torch.tensor(ends, dtype=torch.int32, device="cuda"))
        _check_wgrad(x, x, [max(0, min(ends[0], rows))], "f32", dw[:1])
    torch.cuda.synchronize()


def test_gradients_against_differences():
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    counts = [5, 0, 9, 2]
    x = _randn(g, (16, 24), "f32").requires_grad_()
    w = _randn(g, (4, 24, 10), "f32").requires_grad_()
    dy = _randn(g, (16, 10), "f32")
    ops.expert_linear(x, w, _ends(counts)).backward(dy)

    def value(x, w):
        return sum(float((x[a:b] @ w[e] * dy[a:b].double()).sum()) for e, a, b in _bounds(counts))

    pick = torch.Generator().manual_seed(0)
    for k, leaf in enumerate((x, w)):
        for _ in range(8):
            i = int(torch.randint(leaf.numel(), (), generator=pick))
            args = [t.detach().double().clone() for t in (x, w)]
            flat = args[k].view(-1)
            flat[i] += 1e-3
            up = value(*args)
            flat[i] -= 2e-3
            diff = (up - value(*args)) / 2e-3
            assert abs(float(leaf.grad.reshape(-1)[i]) - diff) <= 1e-4 * (1 + abs(diff))


def test_fp32_matrices_with_bf16_rows():
    """The optimizer's fp32 parameters: rounded for the products, their gradient in fp32."""
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    counts = [64, 100]
    x = _randn(g, (164, 128), "bf16").requires_grad_()
    w = _randn(g, (2, 128, 64), "f32").requires_grad_()
    y = ops.expert_linear(x, w, _ends(counts))
    _check_rows(x.detach(), w.detach().bfloat16(), counts, False, "bf16", y.detach())
    y.backward(y.detach())
    assert w.grad.dtype == torch.float32 and x.grad.dtype == torch.bfloat16
    _check_wgrad(x.detach(), y.detach(), counts, "f32", w.grad)


def test_refusals():
    x = torch.zeros((10, 16), device="cuda")
    w = torch.zeros((2, 16, 8), device="cuda")
    ends = _ends([4, 6])
    for bad in (lambda: tm.expert_matmul(x.cpu(), w, ends), lambda: tm.expert_matmul(x, w[0], ends),
                lambda: tm.expert_matmul(x, w, ends, transposed=True), lambda: tm.expert_matmul(x, w.bfloat16(), ends),
                lambda: tm.expert_matmul(x, w, ends.long()), lambda: tm.expert_matmul(x, w, ends[:1]),
                lambda: tm.expert_matmul(x, w, ends.cpu()), lambda: tm.expert_matmul(x.half(), w.half(), ends),
                lambda: tm.expert_wgrad(x, x[:5], ends), lambda: tm.expert_wgrad(x, x.bfloat16(), ends)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(tm.TurboMuonError) as e:
        tm.expert_wgrad(x, x, ends, dtype=torch.bfloat16)   # fp32 rows, bf16 out
    assert e.value.status == tm.TM_ERR_UNSUPPORTED
    assert tm.expert_matmul(x[:0], w, _ends([0, 0])).shape == (0, 8)
    assert not tm.expert_wgrad(x[:0], x[:0], _ends([0, 0])).any()


# fp32 calls that are large enough for products of bf16 parts: rows, k, n of the rows' products and of the gradient
PARTS = [(2048, 8, 4096), (8, 2048, 4096)]


def _forms(x, w, dy, ends):
    """The rows' product, the same on transposed matrices, and the weight gradient, with their operands."""
    yield "rows", lambda: tm.expert_matmul(x, w, ends)
    yield "transposed", lambda: tm.expert_matmul(dy, w, ends, transposed=True)
    yield "wgrad", lambda: tm.expert_wgrad(x, dy, ends)


@pytest.mark.parametrize("up,down", [(0, 0), (-108, 0), (-122, 60), (-140, 60), (60, -140)])
def test_fp32_parts_keep_small_values(up, down):
    """Values whose last bits lie below the smallest bf16 keep the accuracy of fp32, in every form."""
    log(f"case: fp32 products of values of 2^{up} and 2^{down}")
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    for rows, k, n in PARTS:
        x = (_randn(g, (rows, k), "f32").double() * 2.0 ** up).float()
        w = (_randn(g, (1, k, n), "f32").double() * 2.0 ** down).float()
        dy = (_randn(g, (rows, n), "f32").double() * 2.0 ** down).float()
        ends = _ends([rows])
        if rows > k:
            _check_rows(x, w, [rows], False, "f32", tm.expert_matmul(x, w, ends))
            wt = w.transpose(1, 2).contiguous()
            _check_rows(x, wt, [rows], True, "f32", tm.expert_matmul(x, wt, ends, transposed=True))
        else:
            _check_wgrad(x, dy, [rows], "f32", tm.expert_wgrad(x, dy, ends))


def test_fp32_parts_of_products_below_the_largest_value():
    """A product just below the largest fp32, whose high parts multiply to more than it, stays finite; one
    above it becomes an infinity."""
    log("case: fp32 products next to the largest value")
    big = 1.9990 * 2.0 ** 63
    x, w = torch.full((2048, 1), big, device="cuda"), torch.full((1, 1, 4096), 1.9985 * 2.0 ** 63, device="cuda")
    w[0, 0, 7] = 2.0 ** 65
    y = tm.expert_matmul(x, w, _ends([2048]))
    want = float(x[0, 0].double() * w[0, 0, 0].double())
    assert (y[:, 7] == float("inf")).all()
    keep = torch.arange(4096, device="cuda") != 7
    assert ((y[:, keep].double() - want).abs() <= U * want).all()
    dw = tm.expert_wgrad(x[:1].expand(1, 2048).contiguous(), w[0, :, keep], _ends([1]))
    assert ((dw.double() - want).abs() <= U * want).all()


@pytest.mark.parametrize("pad", [float("nan"), float("inf"), 1e-41])
def test_fp32_results_do_not_depend_on_memory_beside_the_operands(pad):
    log(f"case: fp32 products, {pad} beside the operands")
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    for rows, k, n in ((2050, 130, 4093), (131, 2047, 4093)):
        ends = _ends([rows])

        def inside(*shape):
            store = torch.zeros(shape[:-2] + (shape[-2] + 2, shape[-1] + 7), device="cuda")
            view = store[..., 1:-1, 2:-5]
            view.copy_(_randn(g, shape, "f32"))
            return store, view

        stores, (x, w, dy) = zip(*(inside(rows, k), inside(1, k, n), inside(rows, n)))
        ref = [f() for _, f in _forms(x, w, dy, ends)]
        for store, view in zip(stores, (x, w, dy)):
            kept = view.clone()
            store.fill_(pad)
            view.copy_(kept)
        for (name, f), want in zip(_forms(x, w, dy, ends), ref):
            assert torch.equal(f(), want), (name, rows)


def _digits(got, want, K):
    """The bound of test_long_fp32_sums_keep_their_digits, for sums of more than two of their runs."""
    off = float((got.double() - want).norm()) / float(want.norm())
    assert off <= 0.3 * U * (K / 2) ** 0.5, off / (U * (K / 2) ** 0.5)


@pytest.mark.parametrize("experts,skew,rows,k,n", [(63, 1.4, 27080, 256, 192), (20, 1.5, 24000, 130, 201),
                                                   (64, 3.0, 12000, 64, 65), (8, 2.0, 9001, 500, 511)])
def test_long_fp32_sums_of_uneven_groups_keep_their_digits(experts, skew, rows, k, n):
    """One group holds far more rows than the groups do on average."""
    log(f"case: fp32 weight gradient of {rows} rows unevenly over {experts} experts, {k} x {n}")
    g = torch.Generator(device="cuda")
    g.manual_seed(14)
    share = [(e + 1.0) ** -skew for e in range(experts)]
    counts = [int(rows * s / sum(share)) for s in share]
    counts = counts[1:] + counts[:1]                     # the long one is the last
    rows = sum(counts)
    x, dy = _randn(g, (rows, k), "f32"), _randn(g, (rows, n), "f32")
    dw = tm.expert_wgrad(x, dy, _ends(counts))
    _check_wgrad(x, dy, counts, "f32", dw)
    for e, a, b in _bounds(counts):
        if b - a > 2 * 2816:
            _digits(dw[e], x[a:b].double().t() @ dy[a:b].double(), b - a)
    assert max(counts) > 2 * 2816


def test_long_fp32_sums_without_parts_keep_their_digits():
    """Tiles that go back to fp32 products, here for one small value in each row."""
    log("case: long fp32 sums of values without parts")
    g = torch.Generator(device="cuda")
    g.manual_seed(15)
    rows, K, n = 2048, 9000, 4096
    x, w = _randn(g, (rows, K), "f32"), _randn(g, (1, K, n), "f32")
    x[:, 77] = 1.234567e-37
    want = x.double() @ w[0].double()
    _digits(tm.expert_matmul(x, w, _ends([rows])), want, K)
    _digits(tm.expert_matmul(x, w.transpose(1, 2).contiguous(), _ends([rows]), transposed=True), want, K)
    _digits(tm.expert_wgrad(x.t().contiguous(), w[0], _ends([K]))[0], want, K)


@pytest.mark.parametrize("rows,of", [(r, w) for r in ("f32", "bf16") for w in ("bfloat16", "float16", "float32", "float64")])
def test_matrices_of_another_type(rows, of):
    """What the forward pass takes, the backward pass gives a gradient for, in the matrices' own type:
    the product's, rounded once more."""
    g = torch.Generator(device="cuda")
    g.manual_seed(16)
    counts, wt = [64, 0, 100], getattr(torch, of)
    x = _randn(g, (164, 48), rows).requires_grad_()
    w = (torch.randn((3, 48, 40), generator=g, device="cuda") * 0.1).to(wt).requires_grad_()
    y = ops.expert_linear(x, w, _ends(counts))
    _check_rows(x.detach(), w.detach().to(DT[rows]), counts, False, rows, y.detach())
    y.backward(torch.ones_like(y))
    assert w.grad.dtype is wt and x.grad.dtype is DT[rows]
    for e, a, b in _bounds(counts):
        dy = torch.ones((b - a, 40), dtype=torch.float64, device="cuda")
        want, terms = x.detach()[a:b].double().t() @ dy, x.detach()[a:b].double().abs().t() @ dy
        bound = 2 * (b - a) * U * terms
        eps = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}.get(of, U)
        assert ((w.grad[e].double() - want).abs() <= bound + eps * (want.abs() + bound) + 2.0 ** -25).all()
    _check_rows(torch.ones_like(y), w.detach().to(DT[rows]), counts, True, rows, x.grad)
