"""Sizes and shapes of the training operators at which a launch, a loop or a sum behaves in another way (needs an MI355X)."""
import pytest
import torch

from paper_2110_08450_amd import binding as smfg

from test_gpu_training_ops import BF16, DEV, F16, F32, check, count, norm_grad_of, norm_inputs, norm_of, rounded, strided

pytestmark = pytest.mark.gpu


def test_gradient_of_more_than_2_30_ids():
    """The blocks that add up take three launches.  2^20 ones to a row: every sum is exact; the last row has 77."""
    each, last = 2 ** 20, 77
    n = 2 ** 30 + 5 * each + last
    rows = n // each + 1
    ids = torch.arange(n - 1, -1, -1, device=DEV).div_(each, rounding_mode="floor").to(torch.int32)
    dy = torch.ones((n, 1), dtype=F16, device=DEV)
    want = torch.full((rows, 1), float(each), device=DEV)
    want[rows - 1] = last
    ws = smfg.embedding_grad_workspace(n, rows, 1)
    g = torch.full((rows, 1), 9.0, device=DEV)
    smfg.embedding_grad(ids, count(n), n, dy, g, ws)
    assert torch.equal(g, want)
    smfg.embedding_grad(ids, count(n), n, dy, g, ws, scale=2.0, accumulate=True)
    assert torch.equal(g, 3 * want)
    row_ids, num = torch.full((n,), -7, dtype=torch.int32, device=DEV), count(-1)
    c = torch.full((n, 1), 5.0, dtype=F16, device=DEV)
    smfg.embedding_grad_rows(ids, count(n), n, dy, rows, row_ids, num, c, ws, scale=2.0 ** -12)
    assert int(num) == rows and torch.equal(row_ids[:rows].cpu(), torch.arange(rows, dtype=torch.int32)) and bool((row_ids[rows:] == -7).all())
    assert torch.equal(c[:rows], (want * 2.0 ** -12).half()) and bool((c[rows:] == 5).all())


@pytest.mark.parametrize("n", [0, 3, 300])
def test_gradient_of_a_table_of_2_31_rows(n):
    """All rows that no id names become zeros, beside up to 256 ids by more blocks than a launch has."""
    rows, dim = 2 ** 31 - 1, 2
    at = torch.tensor([0, 2 ** 30 + 1, rows - 1], device=DEV)
    g = torch.ones((rows, dim), dtype=F16, device=DEV)
    ids = at[torch.arange(max(1, n), device=DEV) % 3]
    dy = torch.ones((max(1, n), dim), dtype=F16, device=DEV)
    smfg.embedding_grad(ids, count(n), n, dy, g, smfg.embedding_grad_workspace(n, rows, dim))
    assert torch.equal(g[at], torch.full((3, dim), n / 3, dtype=F16, device=DEV))
    g[at] = 0
    for piece in g.split(2 ** 28):
        assert int(torch.count_nonzero(piece)) == 0


# ---- long rows ----------------------------------------------------------------------------------

U = 2.0 ** -24
LONG = [(20_480, F32, 100.1, 0.0), (65_536, F32, 100.1, 0.0), (2 ** 20, F32, 100.1, 0.0), (2 ** 20, F32, 1.1, 0.0), (2 ** 20 + 3, BF16, 100.1, 0.0),
        (2 ** 20 + 5, F16, 1.1, 0.0), (65_539, F32, 1000.0, 1.0), (2 ** 20, F32, -100.1, 0.5), (65_536, F16, 30.0, 0.5), (20_000, BF16, -1.1, 0.1)]


@pytest.mark.parametrize("dim,dtype,centre,spread", LONG)
def test_layer_norm_of_long_rows_off_centre(dim, dtype, centre, spread):
    """Whatever the row's length, a mean is off by its one rounding to float, dm; the centred values by it and theirs; the variance by dm^2 and two
    roundings of each value; 1 / sqrt(variance + eps) by four more."""
    n, eps = 5, 1e-5
    x = (centre + spread * torch.randn((n, dim), device=DEV, generator=torch.Generator(device=DEV).manual_seed(dim))).to(dtype)
    w, b = torch.full((dim,), 1.5, device=DEV), torch.linspace(-1, 1, dim, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    smfg.layer_norm(x, count(n), n, w, b, eps, y, mean, rstd)
    xd = x.double()
    m = xd.mean(1, keepdim=True)
    d = xd - m
    var = (d * d).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    dm = 1.001 * U * m.abs()
    share = 6 * U + dm * dm / (2 * (var + eps))
    want = d * r * w.double() + b.double()
    tol = 1.5 * r * dm * (1 + share) + (want - b.double()).abs() * (share + 4 * U) + U * (want.abs() + b.double().abs())
    check(y, want, rounded(1.01 * tol, want, dtype))
    check(mean, m[:, 0], dm[:, 0])
    check(rstd, r[:, 0], (r * share)[:, 0] * 1.01)


@pytest.mark.parametrize("dim,dtype,centre,spread", LONG)
def test_layer_norm_grad_of_long_rows_off_centre(dim, dtype, centre, spread):
    """The same of the input's gradient, where dy is far off centre: products and differences are rounded once each, the means once more, whatever
    the row's length."""
    n = 5
    g = torch.Generator(device=DEV).manual_seed(dim)
    dy = (centre + spread * torch.randn((n, dim), device=DEV, generator=g)).to(dtype)
    x = (0.3 + torch.randn((n, dim), device=DEV, generator=g)).to(dtype)
    w = 1 + 0.25 * torch.rand(dim, device=DEV, generator=g) if spread else torch.ones(dim, device=DEV)
    var, mean = torch.var_mean(x.float(), 1, correction=0)
    rstd = (var + 1e-5).rsqrt()
    dx = torch.empty_like(x)
    smfg.layer_norm_grad(dy, x, count(n), n, w, mean, rstd, dx, None, None, None)
    m, r = mean.double()[:, None], rstd.double()[:, None]
    h, gw = (x.double() - m) * r, dy.double() * w.double()
    c1, c2, both = gw.mean(1, keepdim=True), (gw * h).mean(1, keepdim=True), (gw * h).abs().mean(1, keepdim=True)
    want = r * (gw - c1 - h * c2)
    tol = U * (gw.abs() + gw.abs().mean(1, keepdim=True) + c1.abs() + h.abs() * (4 * both + c2.abs()) + 3 * (h * c2).abs()
               + 2 * (gw.abs() + c1.abs() + (h * c2).abs()))
    check(dx, want, rounded(1.01 * (r * tol + U * want.abs()), want, dtype))


# ---- clipping -----------------------------------------------------------------------------------

@pytest.mark.parametrize("scale", [1.0, 0.5])
@pytest.mark.parametrize("tensors,numel", [(2, 10), (90, 3000), (3, 1_000_000)])
def test_no_limit_lets_a_nan_through_and_clips_nothing_else(tensors, numel, scale):
    """max_norm infinite: a NaN makes everything NaN, in place and into other buffers; an infinite norm leaves finite gradients what they are."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        for in_place in (True, False):
            grads = [torch.full((numel,), 3.0, dtype=(F32, F16, BF16)[i % 3], device=DEV) for i in range(tensors)]
            grads[tensors // 2][numel - 1] = bad
            outs = [None if in_place else torch.full((numel,), 7.0, device=DEV) for _ in grads]
            norm = torch.zeros(1, device=DEV)
            smfg.clip_grad_norm(smfg.grad_list(grads, outs), float("inf"), norm, scale=scale)
            got = torch.cat([(g if o is None else o).float() for g, o in zip(grads, outs)])
            if bad != bad:
                assert norm.isnan().all() and got.isnan().all()
            else:
                want = torch.full_like(got, 3.0 * scale)
                want[tensors // 2 * numel + numel - 1] = bad
                assert float(norm) == float("inf") and torch.equal(got, want)


@pytest.mark.parametrize("numel,value,limit,scale", [(10, 1e38, 1e-6, 1.0), (3_000_000, 3e38, 1e-3, 0.25), (1000, -2e35, 1e-9, 4.0), (5, 1e30, 1e-20, 1.0),
                                                     (70_000, 1e20, 1e-12, 1.0), (100, 3e38, 1e-38, 1.0), (9, 3.0, 1e-30, 1.0), (9, 1e-3, 1.0, 2.0 ** -110)])
def test_clipping_of_norms_that_leave_a_float_no_digits_for_the_factor(numel, value, limit, scale):
    """A clipped value has the factor's rounding, the product's and the output's, also where the factor itself is below a float's normal range."""
    g = torch.full((numel,), value, device=DEV) * torch.linspace(0.5, 1, numel, device=DEV)
    small = torch.tensor([1e-30, value * 1e-12], device=DEV)
    b = (torch.ones(numel, device=DEV) * min(abs(value), 1e38)).to(BF16)
    out = torch.zeros(numel, device=DEV)
    total = torch.cat([g, small, b.float()]).double() * scale
    n64 = float(torch.linalg.vector_norm(total))
    factor = scale * min(1.0, limit / (n64 + 1e-6))
    want = [t.double() * factor for t in (g, small, b)]
    norm = torch.zeros(1, device=DEV)
    smfg.clip_grad_norm(smfg.grad_list([g, small, b], [None, None, out]), limit, norm, scale=scale)
    for got, w in zip((g, small, out), want):
        check(got, w, rounded(4 * U * w.abs(), w, F32))


# ---- more rows than a launch has at once ---------------------------------------------------------
#
# k_layer_norm has at most 2048 blocks, k_layer_norm_grad 1024 slices, k_norm_grad_columns 64: every shape of a row's lanes with several rows to
# each of them, the count ending between two blocks' turns.
MANY = [(70_001, 3, F32, F32, 1), (140_007, 31, F16, F32, 2), (200_000, 32, F16, F16, 0), (70_003, 57, BF16, F32, 0), (70_000, 64, F16, F32, 3), (70_000, 100, F16, F32, 0),
        (40_001, 64, F32, F32, 0), (20_005, 250, BF16, BF16, 1), (20_000, 200, F32, F32, 0), (20_000, 1024, F16, F32, 0), (9001, 512, F32, F32, 5), (5000, 2048, F16, F16, 0),
        (5003, 1500, F32, F32, 0), (5000, 4096, BF16, F32, 0), (4500, 6143, F16, F32, 0), (5000, 8192, F16, F16, 0), (4400, 7001, F32, F32, 1), (4300, 12_288, BF16, F32, 0),
        (4200, 16_384, F16, F32, 0), (4200, 8192, F32, F32, 0), (3000, 8193, F32, F32, 1), (2500, 20_001, F16, F32, 0), (300, 16_385, BF16, BF16, 2)]


@pytest.mark.parametrize("cap,dim,dtype,ptype,pad", MANY)
def test_layer_norm_of_many_rows(cap, dim, dtype, ptype, pad):
    n = cap - cap // 37 - 1
    x, w, b = norm_inputs(n, cap, dim, dtype, ptype, pad)
    y, wide = strided((cap, dim), dtype, pad, 5)
    before = wide.clone()
    mean, rstd = torch.full((cap,), 7.0, device=DEV), torch.full((cap,), 7.0, device=DEV)
    smfg.layer_norm(x, count(n), cap, w, b, 1e-5, y, mean, rstd)
    for at in range(0, n, 1000):
        rows = slice(at, min(n, at + 1000))
        want, m, r, tol, tm, tr = norm_of(x[rows], w, b, 1e-5)
        check(y[rows], want, rounded(tol, want, dtype))
        check(mean[rows], m, rounded(tm, m, F32))
        check(rstd[rows], r, rounded(tr, r, F32))
    assert bool((mean[n:] == 7).all()) and bool((rstd[n:] == 7).all())
    before[:n, :dim] = y[:n]
    assert torch.equal(wide.view(torch.int16), before.view(torch.int16))
    z = x.clone()
    smfg.layer_norm(z, count(n), cap, w, b, 1e-5, z)
    assert torch.equal(z[:n], y[:n]) and torch.equal(z[n:], x[n:])


@pytest.mark.parametrize("cap,dim,dtype,ptype,pad", MANY)
def test_layer_norm_grad_of_many_rows(cap, dim, dtype, ptype, pad):
    """Statistics that make (x - mean) * rstd whole numbers, and whole dy: every sum over the rows is exact, so that no row is left out or counted twice.
    dx into a buffer of its own, and in the place of dy and of x."""
    n = cap - cap // 41 - 1
    g = torch.Generator(device=DEV).manual_seed(dim)

    def whole(*shape, most=2):
        return torch.randint(-most, most + 1, shape, device=DEV, generator=g)

    x, _ = strided((cap, dim), dtype, pad, 1)
    dy, _ = strided((cap, dim), dtype, pad, 2)
    x.copy_(whole(cap, dim))
    dy.copy_(whole(cap, dim, most=1))
    w = (1 + 0.2 * torch.randn(dim, device=DEV, generator=g)).to(ptype)
    mean, rstd = whole(cap, most=1).float(), 2.0 ** whole(cap, most=1).abs().float()
    x[n:], dy[n:], mean[n:] = float("nan"), float("nan"), float("nan")
    ws = smfg.layer_norm_grad_workspace(cap, dim)
    dx, wide = strided((cap, dim), dtype, pad, 7)
    before = wide.clone()
    dw, db = torch.full((dim,), 9.0, device=DEV).to(ptype), torch.full((dim,), 9.0, device=DEV).to(ptype)
    smfg.layer_norm_grad(dy, x, count(n), cap, w, mean, rstd, dx, dw, db, ws)
    sums = torch.zeros((2, dim), dtype=torch.float64, device=DEV)
    for at in range(0, n, 1000):
        rows = slice(at, min(n, at + 1000))
        wx, sw, sb, tx, _, _ = norm_grad_of(dy[rows], x[rows], w, mean[rows], rstd[rows])
        check(dx[rows], wx, rounded(tx, wx, dtype))
        sums += torch.stack([sw, sb])
    assert float(sums.abs().max()) * 8 < 2 ** 24 and cap * 12 < 2 ** 24  # also of magnitudes
    assert torch.equal(dw, sums[0].to(ptype)) and torch.equal(db, sums[1].to(ptype))
    before[:n, :dim] = dx[:n]
    assert torch.equal(wide.view(torch.int16), before.view(torch.int16))
    for which in (0, 1):
        given = [dy.clone(), x.clone()]
        a, b = torch.full_like(dw, 9), torch.full_like(db, 9)
        smfg.layer_norm_grad(given[0], given[1], count(n), cap, w, mean, rstd, given[which], a, b, ws)
        assert torch.equal(given[which][:n], dx[:n]) and bool(given[which][n:].isnan().all())
        assert torch.equal(a, dw) and torch.equal(b, db)


@pytest.mark.parametrize("n,spare,dim,dtype,ptype,pad", [(9, 1, 8194, F16, F32, 0), (7, 0, 10_000, BF16, BF16, 1), (5, 2, 12_289, F16, F16, 3), (4, 0, 12_288, BF16, F32, 0),
                                                         (5, 0, 16_384, F16, F32, 0), (3, 1, 16_385, BF16, F32, 1), (3, 0, 30_007, F16, F16, 5), (2, 0, 70_000, BF16, F32, 0)])
def test_layer_norm_and_gradient_of_long_half_rows(n, spare, dim, dtype, ptype, pad):
    cap = n + spare
    x, w, b = norm_inputs(n, cap, dim, dtype, ptype, pad)
    y, mean, rstd = torch.full((cap, dim), 4.0, dtype=dtype, device=DEV), torch.zeros(cap, device=DEV), torch.zeros(cap, device=DEV)
    smfg.layer_norm(x, count(n), cap, w, b, 1e-5, y, mean, rstd)
    want, m, r, tol, tm, tr = norm_of(x[:n], w, b, 1e-5)
    check(y[:n], want, rounded(tol, want, dtype))
    check(mean[:n], m, rounded(tm, m, F32))
    check(rstd[:n], r, rounded(tr, r, F32))
    assert bool((y[n:] == 4).all())
    dy, _ = strided((cap, dim), dtype, pad + 1, 6)
    dx, dw, db = torch.full_like(y, 4), torch.empty_like(w), torch.empty_like(w)
    smfg.layer_norm_grad(dy, x, count(n), cap, w, mean, rstd, dx, dw, db, smfg.layer_norm_grad_workspace(cap, dim))
    wx, ww, wb, tx, tw, tb = norm_grad_of(dy[:n], x[:n], w, mean[:n], rstd[:n])
    check(dx[:n], wx, rounded(tx, wx, dtype))
    check(dw, ww, rounded(tw, ww, ptype))
    check(db, wb, rounded(tb, wb, ptype))
    assert bool((dx[n:] == 4).all())
    z = x.clone()  # dx in the place of x, without the sums
    smfg.layer_norm_grad(dy, z, count(n), cap, w, mean, rstd, z, None, None, None)
    assert torch.equal(z[:n], dx[:n]) and torch.equal(z[n:], x[n:])


@pytest.mark.parametrize("n,rows,dim,dtype,pad", [(600, 5000, 3, F16, 5), (8000, 16_001, 1, F32, 3), (20_000, 50_000, 3, BF16, 2), (20_000, 50_001, 1, F32, 1),
                                                  (9000, 70_000, 7, F16, 1), (300_000, 600_001, 1, F16, 1)])
def test_gradient_of_narrow_rows_apart(n, rows, dim, dtype, pad):
    """Rows shorter than a vector in a wider buffer, cleared beside the sort: what is between them stays."""
    ids = torch.randint(-1, rows, (n,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(n))
    dy = torch.ones((n, dim), dtype=dtype, device=DEV)
    g, wide = strided((rows, dim), dtype, pad, 7)
    before = wide.clone()
    smfg.embedding_grad(ids, count(n), n, dy, g, smfg.embedding_grad_workspace(n, rows, dim))
    before[:, :dim] = torch.bincount(ids[ids >= 0], minlength=rows)[:, None].to(dtype)
    assert torch.equal(wide.view(torch.int16), before.view(torch.int16))
