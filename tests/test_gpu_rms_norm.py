"""Root-mean-square norm, its 8-bit outputs and its gradient against their definitions in 64 bits."""
import pytest
import torch

from paper_2110_08450_amd import binding as smfg

from test_gpu_training_ops import BF16, DEV, F16, F32, U, check, count, depth, gen, rounded, strided

pytestmark = pytest.mark.gpu
I8, E4M3 = torch.int8, torch.float8_e4m3fn
TOP = {I8: 127.0, E4M3: 448.0}

# n, spare rows, dim, type, type of the weight, columns between rows, with a residual
NORMS = [(1, 0, 1, F32, F32, 0, True), (3, 1, 3, F16, F16, 2, True), (17, 0, 7, BF16, F32, 0, False), (100, 20, 8, F16, F32, 0, True), (33, 0, 31, F32, F32, 1, True),
         (65, 3, 64, F32, F32, 0, False), (1000, 24, 100, F16, F16, 0, True), (257, 0, 128, F32, F32, 4, True), (130, 0, 129, BF16, BF16, 0, True),
         (700, 9, 256, F16, F32, 0, True), (90, 0, 257, F32, F32, 3, False), (64, 1, 301, F16, F16, 19, True), (50, 0, 512, BF16, F32, 0, True),
         (41, 0, 513, F32, F32, 0, True), (30, 2, 1000, F16, F16, 0, True), (29, 0, 1025, F32, F32, 0, True), (28, 0, 2048, BF16, BF16, 0, True),
         (27, 1, 2049, F16, F32, 5, True), (26, 0, 4096, BF16, BF16, 0, True), (25, 0, 4099, F32, F32, 0, False), (12, 0, 8192, F16, F32, 0, True),
         (11, 1, 8192, F32, F32, 0, True), (9, 0, 8193, BF16, BF16, 1, True), (5, 0, 20_001, F32, F32, 0, True), (4, 1, 20_003, BF16, BF16, 1, True),
         (1, 4, 5120, BF16, F32, 0, True), (20_000, 0, 100, F32, F32, 0, True), (0, 5, 64, F32, F32, 0, True), (70_000, 3, 20, BF16, F32, 4, True),
         (3, 0, 30_000, F16, F16, 0, False)]


def inputs(n, spare, dim, dtype, ptype, pad, res):
    cap = n + spare
    x, _ = strided((cap, dim), dtype, pad, 1, 2.0)
    r, _ = strided((cap, dim), dtype, pad + 1, 2, 3.0)
    w = (1 + 0.2 * torch.randn(dim, device=DEV, generator=gen(3))).to(ptype)
    return cap, x, r if res else None, w


def norm_of(t, w, eps):
    """(y, r, their tolerances before a rounding) in 64 bits: a sum of squares of one sign, half its relative error in the root, root and inverse."""
    t, w = t.double(), w.double()
    r = 1 / torch.sqrt((t * t).mean(1, keepdim=True) + eps)
    y = t * r * w
    share = ((depth(t.shape[1]) + 4) / 2 + 4) * U
    return y, r[:, 0], (share + 2 * U) * y.abs(), (share * r)[:, 0]


@pytest.mark.parametrize("n,spare,dim,dtype,ptype,pad,res", NORMS)
def test_rms_norm(n, spare, dim, dtype, ptype, pad, res):
    eps = 1e-5
    cap, x, r, w = inputs(n, spare, dim, dtype, ptype, pad, res)
    y, wide = strided((cap, dim), dtype, pad + 1, 5)
    t, wide_t = strided((cap, dim), dtype, pad + 2, 6)
    before, before_t = wide.clone(), wide_t.clone()
    rstd = torch.full((cap,), 7.0, device=DEV)
    smfg.rms_norm(x, count(n), cap, w, eps, y, residual=r, total=t if res else None, rstd=rstd)
    total = (x.float() + r.float()).to(dtype) if res else x
    want, rs, tol, tr = norm_of(total[:n], w, eps)
    check(y[:n], want, rounded(tol, want, dtype))
    check(rstd[:n], rs, rounded(tr, rs, F32))
    assert bool((rstd[n:] == 7).all())
    before[:n, :dim] = y[:n]
    if res:
        before_t[:n, :dim] = total[:n]
    assert torch.equal(wide.view(torch.int16), before.view(torch.int16)) and torch.equal(wide_t.view(torch.int16), before_t.view(torch.int16))
    # the sum and the norm in the place of either input; without the sum; without a weight
    for where in ("x", "residual") if res else ("x",):
        for kept in (False, True):
            a, b = x.clone(), r.clone() if res else None
            here, other = (a, b) if where == "x" else (b, a)
            z = torch.full_like(x, 3.0)
            if kept and res:
                smfg.rms_norm(a, count(n), cap, w, eps, z, residual=b, total=here)
                assert torch.equal(here[:n], total[:n]) and torch.equal(z[:n], y[:n])
                smfg.rms_norm(x, count(n), cap, w, eps, here.copy_(x if where == "x" else r), residual=r, total=z)
                assert torch.equal(z[:n], total[:n])
                a, b = x.clone(), r.clone()
                here = a if where == "x" else b
                smfg.rms_norm(a, count(n), cap, w, eps, here, residual=b, total=b if where == "x" else a)
                assert torch.equal((b if where == "x" else a)[:n], total[:n])
            else:
                smfg.rms_norm(a, count(n), cap, w, eps, here, residual=b)
            assert torch.equal(here[:n], y[:n]) and torch.equal(here[n:], (x if where == "x" else r)[n:])
    z = torch.empty_like(x)
    smfg.rms_norm(x, count(n), cap, None, eps, z, residual=r)
    want, _, tol, _ = norm_of(total[:n], torch.ones_like(w), eps)
    check(z[:n], want, rounded(tol, want, dtype))


@pytest.mark.parametrize("out", [I8, E4M3])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("n,spare,dim,dtype,ptype,pad,res", NORMS)
def test_bytes(n, spare, dim, dtype, ptype, pad, res, group, out):
    """The kept value is off by half a step of its scale (1 / 2 of a whole number; 2^-4 of a float, 2^-10 at least), by the scale's and the factor's
    roundings (4 of them on up to 127 or 448 steps), and by what the norm is."""
    eps = 1e-6
    cap, x, r, w = inputs(n, spare, dim, dtype, ptype, pad, res)
    groups = -(-dim // group) if group else 1
    wide = torch.full((max(1, cap), dim + 3), 85, dtype=torch.uint8, device=DEV)
    y = wide.view(out)[:cap, :dim]
    scales, wide_s = strided((cap, groups), F32, 2, 7)
    before, before_s = wide.clone(), wide_s.clone()
    total = torch.empty_like(x) if res else None
    smfg.rms_norm(x, count(n), cap, w, eps, y, residual=r, total=total, scales=scales, group=group)
    t = (x.float() + r.float()).to(dtype) if res else x
    if res:
        assert torch.equal(total[:n], t[:n])
    want, _, tol, _ = norm_of(t[:n], w, eps)
    width = group or dim
    tops = torch.zeros((n, groups * width), dtype=torch.float64, device=DEV)
    tops[:, :dim] = want.abs()
    top = tops.view(n, groups, width).amax(2) if n else tops.view(0, groups)
    tols = torch.zeros((n, groups * width), dtype=torch.float64, device=DEV)
    tols[:, :dim] = tol
    s = scales[:n].double()
    most = tols.view(n, groups, width).amax(2) if n else top
    check(s, top / TOP[out], (most * 1.01 + U * top) / TOP[out])
    of = torch.repeat_interleave(s, width, 1)[:, :dim]
    q = y[:n].to(F32).double()
    assert bool((q.abs() <= TOP[out]).all())
    half = torch.full_like(q, 0.5) if out == I8 else (want.abs() / of * 2.0 ** -4 * 1.001).nan_to_num(0.0).clamp(min=2.0 ** -10)
    check(q * of, want, tol * 1.01 + of * (half + 4 * U * TOP[out]))
    if n:  # every group has its largest value at the end of the range
        full = torch.zeros((n, groups * width), dtype=torch.float64, device=DEV)
        full[:, :dim] = q.abs()
        assert bool((full.view(n, groups, width).amax(2) == TOP[out]).all())
    before[:n, :dim] = wide[:n, :dim]
    before_s[:n, :groups] = scales[:n]
    assert torch.equal(wide, before) and torch.equal(wide_s.view(torch.int32), before_s.view(torch.int32))


def test_bytes_are_rounded_as_torch_rounds():
    """The same float operations by torch: every value is what torch rounds it to, subnormal ones and zeros of either sign among them."""
    for out in (I8, E4M3):
        dim = 4096
        y = torch.linspace(-TOP[out], TOP[out], dim, device=DEV)
        y[2::5] *= 2.0 ** -12
        y[5] = -0.0
        q, s, rstd = torch.zeros((1, dim), dtype=torch.uint8, device=DEV).view(out), torch.zeros((1, 1), device=DEV), torch.zeros(1, device=DEV)
        smfg.rms_norm(y[None], count(1), 1, torch.ones(dim, device=DEV), 1e-5, q, scales=s, rstd=rstd)
        z = y * rstd  # one rounding, as in the kernel
        want = z * (TOP[out] / z.abs().max())
        want = torch.round(want).to(I8) if out == I8 else want.to(out)
        assert torch.equal(q.view(torch.uint8)[0], want.view(torch.uint8))


def test_rows_of_zeros_infinities_and_nan():
    """A row of zeros has scales of 0; an infinite or NaN row has scales of NaN and harms no other."""
    for dim in (5, 100, 1000, 9000, 20_000):
        x = torch.randn((6, dim), device=DEV, generator=gen(1))
        x[1], x[2, 0], x[4, dim - 1] = 0.0, float("inf"), float("nan")
        y, rstd = torch.empty_like(x), torch.empty(6, device=DEV)
        smfg.rms_norm(x, count(6), 6, None, 1e-5, y, rstd=rstd)
        want, _, tol, _ = norm_of(x[[0, 3, 5]], torch.ones(dim, device=DEV), 1e-5)
        check(y[[0, 3, 5]], want, rounded(tol, want, F32))
        assert not y[1].any() and y[4].isnan().all() and y[2, 0].isnan() and not y[2, 1:].any() and rstd[2] == 0 and rstd[4].isnan()
        for out in (I8, E4M3):
            for group in (0, 32, 128):
                groups = -(-dim // group) if group else 1
                q, s = torch.zeros((6, dim), dtype=torch.uint8, device=DEV).view(out), torch.full((6, groups), 9.0, device=DEV)
                smfg.rms_norm(x, count(6), 6, None, 1e-5, q, scales=s, group=group)
                assert not s[1].any() and not q[1].float().any() and s[4].isnan().all() and not q[4].float().any() and s[2, 0].isnan() and not q[2].float().any()
                assert bool((s[[0, 3, 5]] > 0).all()) and bool(s[[0, 3, 5]].isfinite().all())
        # a weight with a NaN: that column's group alone
        w = torch.ones(dim, device=DEV)
        w[0] = float("nan")
        q, s = torch.zeros((6, dim), dtype=I8, device=DEV), torch.zeros((6, -(-dim // 32)), device=DEV)
        smfg.rms_norm(x, count(6), 6, w, 1e-5, q, scales=s, group=32)
        assert s[0, 0].isnan() and bool(s[0, 1:].isfinite().all())


@pytest.mark.parametrize("n,max_rows", [(-5, 100), (100, 50), (2 ** 40, 300)])
def test_counts_are_held_to_the_launch(n, max_rows):
    x = torch.randn((max_rows + 7, 48), device=DEV, generator=gen(1))
    y, t = torch.full_like(x, 5.0), torch.full_like(x, 5.0)
    smfg.rms_norm(x, count(n), max_rows, None, 1e-5, y, residual=x, total=t)
    m = 0 if n < 0 else max_rows
    assert torch.equal(t[:m], 2 * x[:m]) and bool((y[m:] == 5).all()) and bool((t[m:] == 5).all()) and not bool((y[:m] == 5).all(1).any())
    rstd = torch.ones(max_rows + 7, device=DEV)
    dx, dw, ws = torch.full_like(x, 5.0), torch.empty(48, device=DEV), smfg.rms_norm_grad_workspace(max_rows, 48)
    smfg.rms_norm_grad(x, x, count(n), max_rows, None, rstd, dx, dw, ws)
    assert bool((dx[m:] == 5).all()) and bool(dw.isfinite().all()) and bool((dw == 0).all()) == (m == 0)


def test_rows_2_31_elements_apart():
    """Row offsets pass 32 bits in elements and in bytes, of every matrix."""
    n, dim, apart = 3, 72, 2 ** 31 + 8
    bufs = [torch.empty((n - 1) * apart + dim, dtype=F16, device=DEV) for _ in range(2)]
    x, t = [b.as_strided((n, dim), (apart, 1)) for b in bufs]
    a, b, dy = [torch.randn((n, dim), device=DEV, generator=gen(s)).half() for s in (1, 2, 3)]
    x.copy_(a)
    y, y2, rstd = torch.empty_like(a), torch.empty_like(a), torch.empty(n, device=DEV)
    smfg.rms_norm(x, count(n), n, None, 1e-5, y, residual=b, total=t, rstd=rstd)
    total = (a.float() + b.float()).half()
    smfg.rms_norm(a, count(n), n, None, 1e-5, y2, residual=b)
    assert torch.equal(t, total) and torch.equal(y, y2)
    dx, dx2 = torch.empty_like(a), torch.empty_like(a)
    smfg.rms_norm_grad(dy, total, count(n), n, None, rstd, dx, None, None, grad_total=b)
    x.copy_(b)
    smfg.rms_norm_grad(dy, t, count(n), n, None, rstd, x, None, None, grad_total=x)
    assert torch.equal(x, dx)
    smfg.rms_norm(b, count(n), n, None, 1e-5, t, residual=a)
    smfg.rms_norm(b, count(n), n, None, 1e-5, dx2, residual=a)
    assert torch.equal(t, dx2)
    wide = torch.zeros((n - 1) * apart + dim, dtype=torch.int8, device=DEV)
    q, q2, s, s2 = wide.as_strided((n, dim), (apart, 1)), torch.zeros((n, dim), dtype=I8, device=DEV), torch.zeros((n, 3), device=DEV), torch.zeros((n, 3), device=DEV)
    smfg.rms_norm(a, count(n), n, None, 1e-5, q, scales=s, group=32)
    smfg.rms_norm(a, count(n), n, None, 1e-5, q2, scales=s2, group=32)
    assert torch.equal(q, q2) and torch.equal(s, s2)


def grad_of(dy, t, w, r, dt):
    """(dx, dw, their tolerances before a rounding) in 64 bits, for the given statistics."""
    n, dim = t.shape
    dy, t, w, r = dy.double(), t.double(), w.double(), r.double()[:, None]
    h, g = t * r, dy * w
    c2 = (g * h).mean(1, keepdim=True)
    dx = r * (g - h * c2) + (dt.double() if dt is not None else 0)
    e = depth(dim) + 8
    tol = r * (4 * U * g.abs() + h.abs() * (e * U * (g * h).abs().mean(1, keepdim=True) + 6 * U * c2.abs())) + 2 * U * dx.abs()
    return dx, (dy * h).sum(0), 1.01 * tol, (n + 8) * U * (dy * h).abs().sum(0)


@pytest.mark.parametrize("n,spare,dim,dtype,ptype,pad,res", NORMS + [(5000, 0, 4096, F16, F16, 0, True), (3000, 7, 17_000, BF16, F32, 0, True)])
def test_rms_norm_grad(n, spare, dim, dtype, ptype, pad, res):
    cap, t, dt, w = inputs(n, spare, dim, dtype, ptype, pad, res)
    dy, _ = strided((cap, dim), dtype, pad, 9)
    rstd = (t.float().square().mean(1) + 1e-5).rsqrt()
    dx, wide = strided((cap, dim), dtype, pad + 2, 10)
    before = wide.clone()
    dw = torch.empty_like(w)
    ws = smfg.rms_norm_grad_workspace(cap, dim)
    ws.data.fill_(0xA5)
    smfg.rms_norm_grad(dy, t, count(n), cap, w, rstd, dx, dw, ws, grad_total=dt)
    want, ww, tol, tw = grad_of(dy[:n], t[:n], w, rstd[:n], dt[:n] if res else None)
    check(dx[:n], want, rounded(tol, want, dtype))
    check(dw, ww, rounded(tw, ww, ptype))
    before[:n, :dim] = dx[:n]
    assert torch.equal(wide.view(torch.int16), before.view(torch.int16))
    # in the place of each of the inputs; either alone; without a weight
    for place in range(3 if res else 2):
        a = [dy.clone(), t.clone(), dt.clone() if res else None]
        dw2 = torch.empty_like(w)
        smfg.rms_norm_grad(a[0], a[1], count(n), cap, w, rstd, a[place], dw2, ws, grad_total=a[2])
        assert torch.equal(a[place][:n], dx[:n]) and torch.equal(dw2, dw)
    dx2, dw2 = torch.empty_like(dy), torch.empty_like(w)
    smfg.rms_norm_grad(dy, t, count(n), cap, w, rstd, dx2, None, None, grad_total=dt)
    smfg.rms_norm_grad(dy, t, count(n), cap, w, rstd, None, dw2, ws, grad_total=dt)
    assert torch.equal(dx2[:n], dx[:n]) and torch.equal(dw2, dw)
    smfg.rms_norm_grad(dy, t, count(n), cap, None, rstd, dx2, None, None)
    want, _, tol, _ = grad_of(dy[:n], t[:n], torch.ones_like(w), rstd[:n], None)
    check(dx2[:n], want, rounded(tol, want, dtype))


@pytest.mark.parametrize("dim", [24, 300])
def test_gradient_against_differences(dim):
    """Slopes of a weighted sum of outputs and kept sum, in 64 bits, along random directions; the kernel's gradient is off by its own tolerance alone, and
    the difference by h^2 times a third derivative (h = 1e-4 of unit values: below 1e-6 of the slope's terms)."""
    n = 9
    x, r, dy, dt = [torch.randn((n, dim), device=DEV, generator=gen(s)) for s in (1, 2, 3, 4)]
    w = 1 + 0.2 * torch.randn(dim, device=DEV, generator=gen(5))
    y, t, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device=DEV)
    smfg.rms_norm(x, count(n), n, w, 1e-5, y, residual=r, total=t, rstd=rstd)
    dx, dw, ws = torch.empty_like(x), torch.empty_like(w), smfg.rms_norm_grad_workspace(n, dim)
    smfg.rms_norm_grad(dy, t, count(n), n, w, rstd, dx, dw, ws, grad_total=dt)

    def value(x, r, w):
        t = x + r
        return (t * torch.rsqrt((t * t).mean(1, keepdim=True) + 1e-5) * w * dy.double()).sum() + (t * dt.double()).sum()

    base = [a.double() for a in (x, r, w)]
    for which, grad in ((0, dx), (1, dx), (2, dw)):
        v = torch.randn(base[which].shape, device=DEV, generator=gen(20 + which), dtype=torch.float64)
        h = 1e-4
        up, down = [[a + (s * v if i == which else 0) for i, a in enumerate(base)] for s in (h, -h)]
        slope = (value(*up) - value(*down)) / (2 * h)
        size = (grad.double() * v).abs().sum()
        assert abs(slope - (grad.double() * v).sum()) <= (1e-6 + 200 * U) * size


def test_many_rows_and_streams():
    """More rows than the launch has groups, on another stream, twice: the same bits."""
    n, dim = 300_000, 64
    x = torch.randn((n, dim), device=DEV, generator=gen(1)).half()
    outs = []
    side = torch.cuda.Stream()
    for stream in (None, side):
        y, t, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device=DEV)
        dx, dw, ws = torch.empty_like(x), torch.empty(dim, device=DEV), smfg.rms_norm_grad_workspace(n, dim)
        num = count(n)
        side.wait_stream(torch.cuda.current_stream())
        smfg.rms_norm(x, num, n, None, 1e-5, y, residual=x, total=t, rstd=rstd, stream=stream)
        smfg.rms_norm_grad(y, t, num, n, None, rstd, dx, dw, ws, grad_total=x, stream=stream)
        torch.cuda.synchronize()
        outs.append((y, t, rstd, dx, dw))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    want, rs, tol, _ = norm_of(outs[0][1], torch.ones(dim, device=DEV), 1e-5)
    check(outs[0][0], want, rounded(tol, want, F16))


@pytest.mark.parametrize("out,least", [(I8, 2.0 ** -120), (E4M3, 2.0 ** -119)])
@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("dim", [7, 64, 1000, 9000])
def test_bytes_of_groups_of_tiny_values(dim, group, out, least):
    """Down to the largest value that counts as 0 the factor, 127 or 448 divided by the group's largest, is a float.  Rows of ones have the weight as their norm;
    the shares of the largest value lie apart from what two neighbours of 8 bits have in their middle."""
    share = torch.tensor([0.7, -1.0, 0.0, -0.3], device=DEV).repeat(-(-dim // 4))[:dim]
    groups, width = -(-dim // group) if group else 1, group or dim
    q = (share * TOP[out]).round() if out == I8 else (share * TOP[out]).to(E4M3).float()
    for top in (2.0 ** -124, 2.0 ** -121, 2.0 ** -120, 1.5 * 2.0 ** -120, 1.74 * 2.0 ** -120, 1.76 * 2.0 ** -120, 2.0 ** -119, 2.0 ** -100):
        y, s = torch.full((2, dim), 85, dtype=torch.uint8, device=DEV).view(out), torch.full((2, groups), 9.0, device=DEV)
        smfg.rms_norm(torch.ones((2, dim), device=DEV), count(2), 2, share * top, 0.0, y, scales=s, group=group)
        if top < least:
            assert not s.any() and not y.float().any()
            continue
        tops = torch.nn.functional.pad(share.abs(), (0, groups * width - dim)).view(groups, width).amax(1) * top
        assert bool((tops == top).all())
        # one rounding; a scale below a float's normal range has the steps of its least numbers
        check(s, (tops.double() / TOP[out])[None].expand(2, -1), U * s.double() + 2.0 ** -150)
        assert torch.equal(y.float(), q[None].expand(2, -1))
