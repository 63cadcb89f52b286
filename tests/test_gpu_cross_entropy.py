"""Softmax cross entropy and its gradient against their definition in 64 bits."""
import pytest
import torch

from paper_2110_08450_amd import binding as smfg

from test_gpu_training_ops import BF16, DEV, F16, F32, U, check, count, gen, rounded, strided

pytestmark = pytest.mark.gpu
NINF, INF, NAN = float("-inf"), float("inf"), float("nan")

# n, spare rows, classes, type, columns between rows
CASES = [(1, 0, 1, F32, 0), (5, 3, 2, F16, 1), (64, 0, 3, BF16, 0), (300, 0, 7, F16, 2), (17, 2, 8, F16, 0), (100, 0, 16, F32, 0), (257, 5, 31, F32, 3),
         (1024, 0, 172, F16, 0), (33, 0, 255, BF16, 1), (700, 3, 256, F32, 0), (90, 0, 301, F16, 19), (40, 1, 513, F32, 0), (50, 0, 1013, F32, 3),
         (31, 0, 1024, BF16, 0), (29, 0, 2047, F16, 1), (20, 2, 4096, F16, 0), (15, 0, 5000, F32, 0), (11, 0, 8193, BF16, 1), (9, 1, 10_007, F32, 0),
         (8, 0, 16_384, F16, 0), (7, 0, 16_385, F32, 0), (6, 0, 24_577, F16, 1), (5, 0, 28_672, F32, 0), (4, 1, 28_673, F32, 0), (6, 0, 32_001, BF16, 0),
         (600, 0, 50_000, BF16, 0), (4, 0, 57_344, F16, 0), (3, 0, 57_345, BF16, 1), (3, 1, 128_000, BF16, 0), (2, 0, 150_001, F32, 1), (0, 6, 40, F32, 0),
         (20_000, 100, 47, F16, 0), (9000, 0, 5, F32, 0), (30_001, 0, 1, F16, 0)]


def labels_of(n, classes, dtype, seed):
    """Most are classes, the others padding of several kinds."""
    y = torch.randint(0, classes, (n,), device=DEV, generator=gen(seed))
    u = torch.rand(n, device=DEV, generator=gen(seed + 1))
    y = torch.where(u < 0.05, -100, torch.where(u < 0.08, classes, y))
    if dtype == torch.int64:
        y = torch.where((u > 0.95) & (u < 0.97), 2 ** 32 + 1, y)  # not taken for its low half
    return y.to(dtype)


def depth(classes):
    """Roundings that a term goes through in the sum of a row's exponentials: a lane's columns, those of its vectors, lanes and waves."""
    return 96 + classes // 256


def loss_of(x, y, c):
    """(row losses, gradient for the factor c, counted rows, tolerances before a rounding) in 64 bits.  An exponent is off by three roundings of its
    magnitude, a power by two more; a factor of a lane's maximum by as much again.  Powers below 2^-126 are zeros."""
    x = x.double()
    classes = x.shape[1]
    live = (y >= 0) & (y < classes)
    at = torch.where(live, y, 0).long()[:, None]
    d = x - x.amax(1, keepdim=True)
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    off = ((3 * d.abs() + 8) * U).clamp(max=1).nan_to_num(0.0)
    off_s = (e * off).sum(1, keepdim=True) / s + depth(classes) * U + classes * 2.0 ** -126
    p = e / s
    xy = d.gather(1, at)
    row = (torch.log(s) - xy)[:, 0]
    tol_row = (off_s + 3 * U * torch.log(s).abs())[:, 0] + U * (xy.abs()[:, 0] + 2 * row.abs())
    grad = p.scatter_add(1, at, torch.full_like(s, -1.0)) * c
    tol = abs(c) * (p * (off + off_s + 8 * U) + 2.0 ** -125)
    tol = tol.scatter_add(1, at, torch.full_like(s, abs(c) * 3 * U)) * 1.01
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    return (torch.where(live, row, zero), torch.where(live[:, None], grad, zero), int(live.sum()), torch.where(live, tol_row, zero),
            torch.where(live[:, None], tol, zero))


@pytest.mark.parametrize("n,spare,classes,dtype,pad", CASES)
@pytest.mark.parametrize("label", [torch.int32, torch.int64])
def test_cross_entropy(n, spare, classes, dtype, pad, label):
    cap = n + spare
    x, _ = strided((cap, classes), dtype, pad, 1, 3.0)
    y = labels_of(cap, classes, label, 2)
    ws = smfg.cross_entropy_workspace(cap, classes)
    for reduction, scale in (("mean", 8.0), ("sum", 0.5)):
        ws.data.fill_(0xA5)
        dx, wide = strided((cap, classes), dtype, pad + 1, 3)
        before = wide.clone()
        loss, row = torch.full((1,), 7.0, device=DEV), torch.full((cap,), 7.0, device=DEV)
        smfg.cross_entropy(x, y, count(n), cap, loss, ws, grad_logits=dx, row_loss=row, scale=scale, reduction=reduction)
        many = int(((y[:n] >= 0) & (y[:n] < classes)).sum())
        c = scale / max(1, many) if reduction == "mean" else scale
        want, grad, counted, tol_row, tol = loss_of(x[:n], y[:n], c)
        assert counted == many
        share = 1 / max(1, many) if reduction == "mean" else 1
        check(row[:n], want, rounded(tol_row, want, F32))
        # one more rounding of the whole, and one for each row's own loss
        total = want.sum() * share
        check(loss, total[None], ((tol_row + U * want.abs()).sum() * share)[None] + 2 * U * total.abs() + 1e-40)
        check(dx[:n], grad, rounded(tol + U * grad.abs(), grad, dtype))
        assert bool((row[n:] == 7).all())
        before[:n, :classes] = dx[:n]
        assert torch.equal(wide.view(torch.int16), before.view(torch.int16))
        # without the rows' losses and without a gradient; the gradient in the place of the logits
        loss2, z = torch.zeros(1, device=DEV), x.clone()
        smfg.cross_entropy(x, y, count(n), cap, loss2, ws, reduction=reduction)
        assert torch.equal(loss2, loss)
        smfg.cross_entropy(z, y, count(n), cap, loss2, ws, grad_logits=z, scale=scale, reduction=reduction)
        assert torch.equal(z[:n], dx[:n]) and torch.equal(z[n:], x[n:]) and torch.equal(loss2, loss)


@pytest.mark.parametrize("classes", [5, 40, 172, 1000, 6000, 50_000, 70_000])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_masked_logits(classes, dtype):
    """-infinity, and the type's lowest value, have probability 0; what a row without a label holds does not count; a row that has no
    probabilities is NaN, and so is the mean."""
    low = torch.finfo(dtype).min
    x = (torch.randn((9, classes), device=DEV, generator=gen(1)) * 2).to(dtype)
    y = torch.arange(9, device=DEV) % classes
    x[0, 1:] = NINF  # one class is left, which is the label
    x[1, : classes - 1] = low  # the last is left, and is not the label
    x[2, ::2] = NINF
    y[2] = 1
    x[3] = NAN
    x[4] = INF
    x[5] = NINF
    y[3], y[4], y[5] = -1, classes, -100
    x[6] = low  # all alike
    x[7, 0] = NINF
    y[7] = 0
    ws = smfg.cross_entropy_workspace(9, classes)
    loss, row, dx = torch.zeros(1, device=DEV), torch.zeros(9, device=DEV), torch.full_like(x, 3.0)
    smfg.cross_entropy(x, y, count(7), 9, loss, ws, grad_logits=dx, row_loss=row, reduction="sum")
    some = [0, 1, 2, 6]
    want, grad, _, tol_row, tol = loss_of(x[some], y[some], 1.0)
    keep = want.isfinite()
    check(row[some][keep], want[keep], rounded(tol_row, want, F32)[keep])
    check(dx[some], grad, rounded(tol, grad, dtype))
    assert not dx[3:6].any() and not row[3:6].any() and bool((dx[7:] == 3).all())
    assert row[0] == 0 and float(dx[0].abs().max()) == 0
    # a label of probability 0
    smfg.cross_entropy(x[7:8], y[7:8], count(1), 1, loss, ws, grad_logits=dx[7:8], reduction="sum")
    assert loss == INF and dx[7, 0] == -1 and bool(dx[7].isfinite().all())
    # rows without probabilities
    for r in (3, 4, 5):
        y[r] = 0
        smfg.cross_entropy(x[r:r + 1], y[r:r + 1], count(1), 1, loss, ws, grad_logits=dx[r:r + 1])
        assert loss.isnan().all() and dx[r].isnan().all()
    smfg.cross_entropy(x, y, count(9), 9, loss, ws)
    assert loss.isnan().all()
    # no row counts
    smfg.cross_entropy(x, torch.full_like(y, -1), count(9), 9, loss, ws, grad_logits=dx)
    assert loss == 0 and not dx.any()


@pytest.mark.parametrize("offset", [0.0, 3000.0, -20_000.0])
def test_rows_off_centre(offset):
    """Where all logits of a row are large, differences are what counts."""
    for classes in (100, 5000, 60_000):
        x = torch.randn((8, classes), device=DEV, generator=gen(1)) + offset
        y = torch.arange(8, device=DEV)
        loss, row, dx, ws = torch.zeros(1, device=DEV), torch.zeros(8, device=DEV), torch.empty_like(x), smfg.cross_entropy_workspace(8, classes)
        smfg.cross_entropy(x, y, count(8), 8, loss, ws, grad_logits=dx, row_loss=row)
        want, grad, _, tol_row, tol = loss_of(x, y, 1 / 8)
        check(row, want, rounded(tol_row, want, F32))
        check(dx, grad, rounded(tol, grad, F32))
        assert float(tol.max()) < 1e-6


@pytest.mark.parametrize("classes", [9, 700, 20_000])
def test_gradient_against_differences(classes):
    """Slopes of the mean loss in 64 bits along random directions: h^2 times a third derivative of at most one for h = 1e-4, and the kernel's tolerance."""
    n = 6
    x, y = torch.randn((n, classes), device=DEV, generator=gen(1)), labels_of(n, classes, torch.int64, 3)
    y[0] = 2
    loss, dx, ws = torch.zeros(1, device=DEV), torch.empty_like(x), smfg.cross_entropy_workspace(n, classes)
    smfg.cross_entropy(x, y, count(n), n, loss, ws, grad_logits=dx, scale=2.0)
    v = torch.randn((n, classes), device=DEV, generator=gen(5), dtype=torch.float64)
    live = (y >= 0) & (y < classes)

    def value(x):
        return 2.0 * torch.nn.functional.cross_entropy(x[live], y[live])

    h = 1e-4
    slope = (value(x.double() + h * v) - value(x.double() - h * v)) / (2 * h)
    _, _, _, _, tol = loss_of(x, y, 2.0 / int(live.sum()))
    assert abs(slope - (dx.double() * v).sum()) <= ((tol + U * dx.double().abs()) * v.abs()).sum() + 1e-7


@pytest.mark.parametrize("n,max_rows", [(-5, 100), (100, 50), (2 ** 40, 300), (2 ** 40, 20_000)])
def test_counts_are_held_to_the_launch(n, max_rows):
    classes = 24
    x = torch.randn((max_rows + 7, classes), device=DEV, generator=gen(1))
    y = torch.zeros(max_rows + 7, dtype=torch.int32, device=DEV)
    loss, dx, ws = torch.full((1,), 9.0, device=DEV), torch.full_like(x, 5.0), smfg.cross_entropy_workspace(max_rows, classes)
    smfg.cross_entropy(x, y, count(n), max_rows, loss, ws, grad_logits=dx)
    m = 0 if n < 0 else max_rows
    assert bool((dx[m:] == 5).all()) and bool((dx[:m] != 5).all())
    if m == 0:
        assert loss == 0
    else:
        want, grad, _, tol_row, tol = loss_of(x[:m], y[:m], 1 / m)
        check(dx[:m], grad, rounded(tol + U * grad.abs(), grad, F32))
        check(loss, want.mean()[None], ((tol_row + 3 * U * want.abs()).mean())[None])


def test_no_rows_at_all():
    x, y = torch.zeros((0, 7), device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV)
    for reduction in ("mean", "sum"):
        loss = torch.full((1,), 9.0, device=DEV)
        smfg.cross_entropy(x, y, count(0), 0, loss, smfg.cross_entropy_workspace(0, 7), grad_logits=x, reduction=reduction)
        assert loss == 0


def test_rows_2_31_elements_apart():
    n, classes, apart = 3, 72, 2 ** 31 + 8
    buf = torch.empty((n - 1) * apart + classes, dtype=F16, device=DEV)
    x = buf.as_strided((n, classes), (apart, 1))
    a = torch.randn((n, classes), device=DEV, generator=gen(1)).half()
    x.copy_(a)
    y = torch.tensor([3, -1, 71], device=DEV)
    losses, dx, ws = torch.zeros((2, 1), device=DEV), torch.empty_like(a), smfg.cross_entropy_workspace(n, classes)
    smfg.cross_entropy(a, y, count(n), n, losses[0], ws, grad_logits=dx)
    smfg.cross_entropy(x, y, count(n), n, losses[1], ws, grad_logits=x)
    assert torch.equal(losses[0], losses[1]) and torch.equal(x, dx)


def test_logits_of_more_than_2_32_elements():
    """66 000 rows of 65 537 halfs, equal but for one: offsets pass 32 bits within a dense matrix."""
    n, classes = 66_000, 65_537
    x = torch.zeros((n, classes), dtype=F16, device=DEV)
    x[n - 1, 5] = 4.0
    y = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    y[n - 1], y[0] = 5, classes - 1
    loss, ws = torch.zeros(1, device=DEV), smfg.cross_entropy_workspace(n, classes)
    smfg.cross_entropy(x, y, count(n), n, loss, ws, grad_logits=x, reduction="sum", scale=65536.0)
    some = torch.zeros((2, classes), device=DEV)
    some[1, 5] = 4.0
    want, grad, _, tol_row, tol = loss_of(some, y[[0, n - 1]], 65536.0)
    check(loss, want.sum()[None], (tol_row.sum() + 4 * U * want.sum())[None])
    got, large = x[[0, n - 1]], grad.abs() >= 65520  # what rounds to a half's infinity: the label's -65535 of the first row
    assert torch.equal(got[large], grad[large].half()) and int(large.sum()) == 1
    check(got[~large], grad[~large], rounded(tol, grad, F16)[~large])
    assert not x[1].any() and not x[n - 2].any() and not x[n // 2].any()


def test_streams_and_again():
    """The same bits on another stream and a second time, of rows that several blocks share and of those that count in launches of their own."""
    for n, classes in ((9000, 33), (500, 9000), (40, 70_000)):
        x, y = torch.randn((n, classes), device=DEV, generator=gen(1)).half(), labels_of(n, classes, torch.int32, 5)
        side, outs = torch.cuda.Stream(), []
        for stream in (None, side, None):
            loss, row, dx, ws, num = torch.zeros(1, device=DEV), torch.zeros(n, device=DEV), torch.empty_like(x), smfg.cross_entropy_workspace(n, classes), count(n)
            side.wait_stream(torch.cuda.current_stream())
            smfg.cross_entropy(x, y, num, n, loss, ws, grad_logits=dx, row_loss=row, scale=1024.0, stream=stream)
            torch.cuda.synchronize()
            outs.append((loss, row, dx))
        for o in outs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(outs[0], o))


@pytest.mark.parametrize("classes", [1500, 3000, 5000, 20_000, 28_672, 50_000, 57_344, 70_000])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("level", [-80.0, -100.0, -1000.0, -60_000.0])
def test_masked_columns_beside_low_logits(classes, dtype, level):
    """What is left of a row after masking may be far below zero: lanes that hold masked columns alone have no exponential, whatever the row's largest logit is."""
    for masked in (NINF, torch.finfo(dtype).min):
        x = torch.full((5, classes), masked, device=DEV)
        x[0, :40] = torch.randn(40, device=DEV, generator=gen(1)) + level  # the head of a vocabulary
        x[1, -9:] = torch.randn(9, device=DEV, generator=gen(2)) + level  # its end
        x[2, classes // 2] = level  # one class
        x[3, ::2] = torch.randn(len(range(0, classes, 2)), device=DEV, generator=gen(3)) + level
        x[4, :40] = level
        x = x.to(dtype)
        y = torch.tensor([3, classes - 2, classes // 2, 0, -100], device=DEV)
        loss, row, dx, ws = torch.zeros(1, device=DEV), torch.zeros(5, device=DEV), torch.empty_like(x), smfg.cross_entropy_workspace(5, classes)
        smfg.cross_entropy(x, y, count(5), 5, loss, ws, grad_logits=dx, row_loss=row, scale=0.5)
        want, grad, _, tol_row, tol = loss_of(x, y, 0.5 / 4)
        check(row, want, rounded(tol_row, want, F32))
        check(dx, grad, rounded(tol, grad, dtype))
        z = x.clone()
        smfg.cross_entropy(z, y, count(5), 5, loss, ws, grad_logits=z, scale=0.5)
        assert torch.equal(z, dx)
