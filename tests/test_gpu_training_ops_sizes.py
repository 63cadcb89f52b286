"""Sizes and shapes of the training operators at which a launch, a loop or a sum behaves in another way (needs an MI355X)."""
import pytest
import torch

from paper_2110_08450_amd import binding as smfg

from test_gpu_training_ops import BF16, DEV, F16, F32, check, count, rounded

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
