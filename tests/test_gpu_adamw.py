"""AdamW over many tensors and touched rows, with states of 32 and of 8 bits, against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2110_08450_amd import binding as smfg

from test_gpu_training_ops import BF16, DEV, F16, F32, U, check, count, gen, rounded

pytestmark = pytest.mark.gpu
B = smfg.STATE_BLOCK
LR, B1, B2, EPS, WD = 1e-2, 0.9, 0.999, 1e-8, 0.1
TYPES = [(F32, F32, None), (F32, F16, F16), (F32, BF16, BF16), (F32, F16, BF16), (F16, F16, None), (F16, F32, None), (BF16, BF16, None), (BF16, F32, None)]


def values_of(k, scale, cols):
    """(m, sqrt(v)) in 64 bits: a state's numbers with the scales of their row's blocks."""
    s = torch.repeat_interleave(scale.double().reshape(-1, -(-cols // B)), B, 1)[:, :cols].reshape(k.shape)
    x = k.double()
    return (s * x * x.abs() / 127 ** 2) if k.dtype == torch.int8 else s * (x / 255) ** 2


class Tensor:
    """One parameter with its state, as the library has it and in 64 bits."""

    def __init__(self, shape, ptype, gtype, ctype, bytes_, seed, decay=WD, misplaced=0, grad_shape=None):
        def randn(shape, spread, s):
            return torch.randn(shape, device=DEV, generator=gen(100 * seed + s)) * spread

        def place(t):
            """At an odd address, between guards."""
            buf = torch.full((t.numel() + misplaced + 9,), 77, dtype=torch.int32, device=DEV).to(t.dtype)
            buf[misplaced:misplaced + t.numel()] = t.reshape(-1)
            self.guards.append((buf, misplaced, t.numel()))
            return buf[misplaced:misplaced + t.numel()].view(t.shape)

        self.guards, self.decay = [], decay
        self.rows, self.cols = (shape[0], math.prod(shape[1:])) if len(shape) > 1 else (1, math.prod(shape))
        self.p, self.g = place(randn(shape, 1.0, 1).to(ptype)), place((randn(grad_shape or shape, 0.1, 2)).to(gtype))
        self.copy = place(torch.zeros(shape, dtype=ctype, device=DEV)) if ctype is not None else None
        m, u = randn(shape, 0.05, 3), randn(shape, 0.1, 4).abs()
        self.ms = self.vs = None
        if bytes_:
            units = -(-self.cols // B)
            self.m = place(torch.randint(-127, 128, shape, device=DEV, generator=gen(100 * seed + 5)).to(torch.int8))
            self.v = place(torch.randint(0, 256, shape, device=DEV, generator=gen(100 * seed + 6)).to(torch.uint8))
            scale = (self.rows, units) if len(shape) > 1 else (units,)
            self.ms, self.vs = place(randn(scale, 0.1, 7).abs() + 0.01), place(randn(scale, 0.1, 8).abs() + 0.01)
        else:
            self.m, self.v = place(m), place(u * u)

    def state(self):
        if self.ms is None:
            return self.m.double(), self.v.double(), 1 * U, 1 * U
        # numbers of 8 bits become floats: factor, its products
        return values_of(self.m, self.ms, self.cols), values_of(self.v, self.vs, self.cols) ** 2, 8 * U, 14 * U

    def guarded(self):
        return all(bool((b[:a].float() == torch.full((a,), 77, dtype=torch.int32, device=DEV).to(b.dtype).float()).all())
                   and bool((b[a + n:].float() == torch.full((b.numel() - a - n,), 77, dtype=torch.int32, device=DEV).to(b.dtype).float()).all()) for b, a, n in self.guards)


def step_of(p, m, v, g, off_m, off_v, t, f, decay, lr=LR, b1=B1, b2=B2, eps=EPS):
    """(p, m, v, their tolerances before a rounding) in 64 bits.  f, the factor of the gradient, and each coefficient are rounded once, as is each product
    and sum; the corrections are off by some 4 U, root and quotient by 3."""
    p, g = p.double(), g.double() * f
    am, ag, bv, bg = b1 * m, (1 - b1) * g, b2 * v, (1 - b2) * g * g
    m2, v2 = am + ag, bv + bg
    tol_m = (3 * U + off_m) * am.abs() + 6 * U * ag.abs() + 2.0 ** -126
    tol_v = (3 * U + off_v) * bv + 9 * U * bg + 2.0 ** -126
    c1, root = 1 - b1 ** t, math.sqrt(1 - b2 ** t)
    den = v2.sqrt() / root + eps
    upd = lr * m2 / c1 / den
    rel_v = (tol_v / v2.clamp(min=1e-300)).clamp(max=1.0)
    tol_u = lr / c1 / den * tol_m + upd.abs() * (rel_v / 2 + 20 * U)
    new = p - lr * decay * p - upd
    tol_p = 1.01 * tol_u + U * (2 * p.abs() + 6 * (lr * decay * p).abs() + 2 * new.abs()) + 2.0 ** -126
    return new, m2, v2, tol_p, 1.01 * tol_m, 1.01 * tol_v


def check_state(t, m, v, tol_m, tol_v, rows=None):
    """States of 32 bits: the values.  Of 8: the scales are the blocks' largest, and every number is the nearest (half a step in the root, which is off by
    four roundings on up to 127 or 255 steps), or 1 where it would be 0."""
    pick = (lambda x: x) if rows is None else (lambda x: x[rows])
    if t.ms is None:
        check(pick(t.m), m, rounded(tol_m, m, F32))
        check(pick(t.v), v, rounded(tol_v, v, F32))
        return
    units = -(-t.cols // B)

    def tops(x):
        flat = x.reshape(-1, t.cols)
        wide = torch.zeros((flat.shape[0], units * B), dtype=torch.float64, device=DEV)
        wide[:, :t.cols] = flat
        return wide.view(-1, units, B).amax(2)

    root, tol_root = v.sqrt(), tol_v / v.sqrt().clamp(min=1e-150) + 2 * U * v.sqrt()
    for k, s, x, tol, most in ((t.m, t.ms, m.abs(), tol_m, 127), (t.v, t.vs, root, tol_root, 255)):
        k, s = pick(k), pick(s.reshape(-1, units)) if rows is not None else s.reshape(-1, units)
        a = tops(x)
        check(s, a, tops(tol) + U * a)
        wide = torch.repeat_interleave(s.double(), B, 1)[:, :t.cols].reshape(x.shape)
        kk, slack = k.double().abs(), most * 4 * U
        low, high = ((kk - 0.5 - slack).clamp(min=0) / most) ** 2 * wide, ((kk + 0.5 + slack) / most) ** 2 * wide
        if most == 255:
            low = torch.where(kk == 1, 0.0, low)
            assert bool((kk[x > tol] >= 1).all())
        bad = (x < low - tol) | (x > high + tol)
        assert not bad.any(), (int(bad.sum()), kk[bad][:4], x[bad][:4], wide[bad][:4])
        if most == 127:
            assert bool(((torch.sign(k.double()) * torch.sign(m) >= 0) | (m.abs() <= tol_m)).all())


def run(tensors, step=1, **more):
    lst = smfg.adamw_list([t.p for t in tensors], [t.g for t in tensors], [t.m for t in tensors], [t.v for t in tensors],
                          m_scales=[t.ms for t in tensors], v_scales=[t.vs for t in tensors], copies=[t.copy for t in tensors],
                          weight_decay=[t.decay for t in tensors])
    smfg.adamw(lst, step, LR, betas=(B1, B2), eps=EPS, **more)
    return lst


def check_step(t, before, t_step, f, decay, rows=None):
    p, (m, v, om, ov), g = before
    want, wm, wv, tp, tm, tv = step_of(p, m, v, g, om, ov, t_step, f, decay)
    check(t.p if rows is None else t.p[rows], want, rounded(tp, want, t.p.dtype))
    if t.copy is not None:
        check(t.copy if rows is None else t.copy[rows], want, rounded(tp + U * want.abs(), want, t.copy.dtype))
    check_state(t, wm, wv, tm, tv, rows)
    assert t.guarded()


SHAPES = [(1,), (2,), (3,), (4,), (7,), (8,), (127,), (128,), (129,), (1000,), (2049,), (70_000,), (3, 5), (40, 128), (33, 129), (17, 300), (1000, 36), (5, 1)]


@pytest.mark.parametrize("bytes_", [False, True])
@pytest.mark.parametrize("ptype,gtype,ctype", TYPES)
@pytest.mark.parametrize("misplaced", [0, 1])
def test_a_step_of_many_shapes(ptype, gtype, ctype, bytes_, misplaced):
    tensors = [Tensor(s, ptype, gtype, ctype, bytes_, i, decay=0.0 if len(s) == 1 else WD, misplaced=misplaced) for i, s in enumerate(SHAPES)]
    before = [(t.p.clone(), t.state(), t.g.clone()) for t in tensors]
    run(tensors, step=3)
    for t, b in zip(tensors, before):
        check_step(t, b, 3, 1.0, t.decay)
        assert torch.equal(t.g, b[2])


def test_types_and_sizes_together():
    """More tensors than the launch's arguments hold, each of another kind; empty ones among them."""
    tensors = []
    for i in range(150):
        p, g, c = TYPES[i % len(TYPES)]
        tensors.append(Tensor((i * 37 % 5000 + 1,) if i % 7 else (i % 9 + 1, 40 + i), p, g, c, i % 3 == 0, i, decay=0.01 * (i % 4), misplaced=i % 5))
    tensors.insert(20, Tensor((0,), F32, F32, None, False, 7))
    before = [(t.p.clone(), t.state(), t.g.clone()) for t in tensors]
    run(tensors, step=1000)
    for t, b in zip(tensors, before):
        if t.p.numel():
            check_step(t, b, 1000, 1.0, t.decay)


@pytest.mark.parametrize("bytes_", [False, True])
@pytest.mark.parametrize("step", [1, 2, 10, 10 ** 6, 2 ** 40])
def test_steps(bytes_, step):
    """The corrections of the first step and of a late one; the step and the rate from the device."""
    for on_device in (False, True):
        t = Tensor((5000,), F32, F32, None, bytes_, 1)
        before = (t.p.clone(), t.state(), t.g.clone())
        more = dict(device_step=count(step - 1), device_lr=torch.tensor([1.0], device=DEV)) if on_device else {}
        run([t], step=1 if on_device else step, **more)
        check_step(t, before, step, 1.0, WD)


@pytest.mark.parametrize("norm,max_norm,scale", [(0.5, 1.0, 1.0), (8.0, 1.0, 1.0), (8.0, 1.0, 1 / 1024), (1e-3, 1e-4, 3.0), (7.0, float("inf"), 0.5)])
def test_clipping_by_a_norm_at_hand(norm, max_norm, scale):
    for bytes_ in (False, True):
        t = Tensor((3000,), F32, F16, F16, bytes_, 2)
        before = (t.p.clone(), t.state(), t.g.clone())
        n = torch.tensor([norm], device=DEV)
        run([t], step=5, norm=n, max_norm=max_norm, scale=scale)
        check_step(t, before, 5, scale * min(1.0, max_norm / (scale * float(n) + 1e-6)), WD)


def test_factors_below_a_floats_range():
    """Gradients of 1e38 with a limit of 1e-3: the factor has few digits as a float, their product has them all."""
    t = Tensor((1000,), F32, F32, None, False, 3)
    t.g.mul_(1e37)
    before = (t.p.clone(), t.state(), t.g.clone())
    run([t], step=5, norm=torch.tensor([3e38], device=DEV), max_norm=1e-3)
    check_step(t, before, 5, 1e-3 / float(torch.tensor(3e38)), WD)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_no_step_with_a_norm_that_is_not_finite(bad):
    for bytes_ in (False, True):
        for many in (1, 60):
            tensors = [Tensor((500,), F32, F32, F16, bytes_, i) for i in range(many)]
            before = [[x.clone() for x in (t.p, t.m, t.v, t.copy)] for t in tensors]
            run(tensors, norm=torch.tensor([bad], device=DEV), max_norm=1.0)
            for t, b in zip(tensors, before):
                assert all(torch.equal(x, y) for x, y in zip((t.p, t.m, t.v, t.copy), b))


@pytest.mark.parametrize("bytes_", [False, True])
def test_infinite_and_nan_gradients(bytes_):
    """Without a norm they reach their elements alone, and of states of 8 bits their block."""
    t = Tensor((1000,), F32, F32, None, bytes_, 4)
    before = (t.p.clone(), t.state(), t.g.clone())
    t.g[130], t.g[700] = float("nan"), float("inf")
    run([t], step=2)
    want, wm, wv, tp, tm, tv = step_of(*before[:1], *before[1][:2], before[2], *before[1][2:], 2, 1.0, WD)
    fine = torch.ones(1000, dtype=torch.bool, device=DEV)
    fine[[130, 700]] = False
    check(t.p[fine], want[fine], rounded(tp, want, F32)[fine])
    assert t.p[130].isnan() and t.p[700].isnan()  # infinity over infinity
    if bytes_:
        m, v = torch.empty(1000, device=DEV), torch.empty(1000, device=DEV)
        smfg.adamw_values(t.m, t.ms, m)
        smfg.adamw_values(t.v, t.vs, v)
        for x in (m, v):
            assert x[128:256].isnan().all() and x[640:768].isnan().all() and bool(x[:128].isfinite().all()) and bool(x[768:].isfinite().all())


def test_nothing_to_step():
    smfg.adamw(smfg.adamw_list([], [], [], []), 1, LR)
    e = [torch.zeros(0, device=DEV) for _ in range(4)]
    smfg.adamw(smfg.adamw_list([e[0]], [e[1]], [e[2]], [e[3]]), 1, LR)


def test_a_loss_scale_is_undone_with_the_norm_of_the_scaled_gradients():
    """Gradients 1024 times as large, their norm, and a scale of 1 / 1024: the step of the gradients themselves, bit for bit, as powers of two are exact."""
    a, b = Tensor((3000,), F32, F32, None, False, 2), Tensor((3000,), F32, F32, None, False, 2)
    b.g.mul_(1024)
    norm = torch.zeros(1, device=DEV)
    for t, scale in ((a, 1.0), (b, 1 / 1024)):
        before = t.g.clone()
        smfg.clip_grad_norm(smfg.grad_list([t.g]), float("inf"), norm)
        assert torch.equal(t.g, before)
        run([t], step=2, norm=norm, max_norm=0.5, scale=scale)
    assert torch.equal(a.p, b.p) and torch.equal(a.m, b.m) and torch.equal(a.v, b.v)


def test_zeros():
    """Zeroed memory is a state of zeros; a gradient of zeros then moves nothing but by the decay, and leaves zeros."""
    for bytes_ in (False, True):
        t = Tensor((700,), F32, F32, None, bytes_, 5)
        for x in (t.m, t.v, t.ms, t.vs, t.g):
            if x is not None:
                x.zero_()
        p = t.p.clone()
        run([t])
        want = p.double() * (1 - LR * WD)
        check(t.p, want, 3 * U * p.double().abs())
        assert not t.m.any() and not t.v.any() and (t.ms is None or not (t.ms.any() or t.vs.any()))


def test_small_second_moments_are_not_lost():
    """Beside a gradient 10^6 times as large an element's v is kept as the least there is, not as 0: its next step is no larger than its last."""
    t = Tensor((128,), F32, F32, None, True, 6, decay=0.0)
    for x in (t.m, t.v, t.ms, t.vs):
        x.zero_()
    t.g.fill_(1e-6)
    t.g[5] = 1.0
    run([t])
    assert bool((t.v > 0).all()) and t.v[5] == 255
    p = t.p.clone()
    run([t], step=2)
    assert float((t.p - p).abs().max()) <= 1.1 * LR * 2


TABLES = [(1, 1, 1), (5, 9, 3), (50, 300, 4), (200, 1000, 7), (64, 100, 32), (1000, 5000, 100), (77, 90, 127), (300, 400, 128), (200, 777, 129), (31, 40, 301),
          (4000, 4001, 36), (3, 9, 5000), (0, 10, 16), (20_000, 50_000, 64)]


@pytest.mark.parametrize("n,rows,dim", TABLES)
@pytest.mark.parametrize("bytes_", [False, True])
@pytest.mark.parametrize("ptype,gtype,ctype", [TYPES[0], TYPES[2], TYPES[4], TYPES[7]])
def test_touched_rows(n, rows, dim, ptype, gtype, ctype, bytes_):
    """Rows by id; those outside the table are left out, and all others are as they were."""
    spare = 3
    t = Tensor((rows, dim), ptype, gtype, ctype, bytes_, 7, misplaced=n % 2, grad_shape=(n + spare, dim))
    ids = torch.randperm(rows, device=DEV, generator=gen(8))[:n].sort().values.int()
    ids = torch.cat([ids, torch.full((spare,), 0, dtype=torch.int32, device=DEV)])  # what lies behind the count is not read as a row
    if n > 4:
        ids[0], ids[n - 1] = -1, rows
    live = torch.nonzero((ids[:n] >= 0) & (ids[:n] < rows))[:, 0]
    at = ids[live].long()
    m, v, om, ov = t.state()
    before = (t.p[at].clone(), (m[at], v[at], om, ov), t.g[live].clone())
    whole = [x.clone() for x in (t.p, t.m, t.v, t.copy, t.ms, t.vs) if x is not None]
    lst = smfg.adamw_list([t.p], [t.g], [t.m], [t.v], m_scales=[t.ms], v_scales=[t.vs], copies=[t.copy], rows=[count(n)], row_ids=[ids], weight_decay=WD)
    smfg.adamw(lst, 3, LR, betas=(B1, B2), eps=EPS)
    check_step(t, before, 3, 1.0, WD, rows=at)
    rest = torch.ones(rows, dtype=torch.bool, device=DEV)
    rest[at] = False
    for x, y in zip([x for x in (t.p, t.m, t.v, t.copy, t.ms, t.vs) if x is not None], whole):
        assert torch.equal(x[rest], y[rest])


@pytest.mark.parametrize("n,cap", [(-3, 20), (50, 20), (2 ** 40, 20), (0, 20)])
def test_counts_are_held_to_the_gradient(n, cap):
    for by_id in (False, True):
        t = Tensor((cap, 40), F32, F32, None, False, 9)
        p = t.p.clone()
        lst = smfg.adamw_list([t.p], [t.g], [t.m], [t.v], rows=[count(n)], row_ids=[torch.arange(cap, dtype=torch.int32, device=DEV)] if by_id else None)
        smfg.adamw(lst, 1, LR)
        m = max(0, min(n, cap))
        assert torch.equal(t.p[m:], p[m:]) and bool((t.p[:m] != p[:m]).any(1).all())


def test_a_table_beyond_32_bits():
    """Offsets pass 2^32 elements, with states of 8 bits."""
    rows, dim = 40_000_000, 120
    p, m, v = torch.zeros((rows, dim), dtype=F16, device=DEV), torch.zeros((rows, dim), dtype=torch.int8, device=DEV), torch.zeros((rows, dim), dtype=torch.uint8, device=DEV)
    ms, vs = torch.zeros((rows, 1), device=DEV), torch.zeros((rows, 1), device=DEV)
    ids = torch.tensor([0, 35_791_394, 35_791_395, rows - 1], dtype=torch.int32, device=DEV)
    g = torch.randn((4, dim), device=DEV, generator=gen(1)).half()
    lst = smfg.adamw_list([p], [g], [m], [v], [ms], [vs], rows=[count(4)], row_ids=[ids])
    smfg.adamw(lst, 1, LR)
    small = Tensor((4, dim), F16, F16, None, True, 1)
    for x in (small.p, small.m, small.v, small.ms, small.vs):
        x.zero_()
    smfg.adamw(smfg.adamw_list([small.p], [g], [small.m], [small.v], [small.ms], [small.vs]), 1, LR)
    at = ids.long()
    assert torch.equal(p[at], small.p) and torch.equal(m[at], small.m) and torch.equal(v[at], small.v) and torch.equal(ms[at], small.ms) and torch.equal(vs[at], small.vs)
    assert int((ms != 0).sum()) == 4 and not p[1].any() and not p[rows - 2].any()
    # a dense one, as a single row
    flat = [x.reshape(-1) for x in (p, m, v)]
    n = flat[0].numel()
    assert n > 2 ** 32
    gd = torch.zeros(n, dtype=F16, device=DEV)
    gd[n - 1] = 1.0
    scales = [torch.zeros(-(-n // B), device=DEV) for _ in range(2)]
    for x in flat:
        x.zero_()
    smfg.adamw(smfg.adamw_list([flat[0]], [gd], [flat[1]], [flat[2]], [scales[0]], [scales[1]]), 1, LR)
    assert int(torch.count_nonzero(flat[0])) == 1 and flat[0][n - 1] == torch.tensor(-LR).half() and flat[1][n - 1] == 127 and flat[2][n - 1] == 255
    assert int((scales[0] != 0).sum()) == 1 and scales[0][-1] != 0


@pytest.mark.parametrize("shape,by_row", [((1,), False), ((129,), False), ((5000,), False), ((7, 3), True), ((40, 300), True), ((3, 4097), True), ((0,), False)])
@pytest.mark.parametrize("out", [F32, F16, BF16])
def test_values(shape, by_row, out):
    """Each at most five roundings of floats, of which v has its root's twice; then its own."""
    cols = shape[1] if by_row else shape[0]
    units = -(-cols // B)
    s = torch.rand((shape[0], units) if by_row else (units,), device=DEV, generator=gen(1))
    for dtype, low, high in ((torch.int8, -127, 128), (torch.uint8, 0, 256)):
        k = torch.randint(low, high, shape, device=DEV, generator=gen(2)).to(dtype)
        x = torch.full(shape, 9.0, device=DEV).to(out)
        smfg.adamw_values(k, s, x)
        if k.numel():
            want = values_of(k, s, cols)
            want = want if dtype == torch.int8 else want ** 2
            check(x, want, rounded(11 * U * want.abs(), want, out))


def test_many_steps_follow_the_64_bit_ones():
    """A hundred steps on the same data: states of 32 bits stay within what their roundings add up to; those of 8 lead to the minimum of a quadratic as well."""
    n = 4096
    target = torch.randn(n, device=DEV, generator=gen(1))
    for bytes_ in (False, True):
        t = Tensor((n,), F32, F32, None, bytes_, 10, decay=0.0)
        for x in (t.p, t.m, t.v, t.ms, t.vs):
            if x is not None:
                x.zero_()
        p = torch.zeros(n, dtype=torch.float64, device=DEV)
        m, v = torch.zeros_like(p), torch.zeros_like(p)
        lst = smfg.adamw_list([t.p], [t.g], [t.m], [t.v], [t.ms], [t.vs])
        for i in range(1, 301):
            t.g.copy_(t.p - target)
            smfg.adamw(lst, i, LR, betas=(B1, B2), eps=EPS)
            p, m, v, *_ = step_of(p, m, v, p - target.double(), 0, 0, i, 1.0, 0.0)
        exact = float((p - target.double()).norm())
        mine = float((t.p.double() - target.double()).norm())
        if not bytes_:
            # each step adds some 30 roundings of a step of LR at most, and one of p; errors of p shrink on the way to the minimum
            assert float((t.p.double() - p).abs().max()) <= 300 * (40 * U * LR * 8 + 2 * U * 8)
        else:
            assert mine <= 0.2 * float(target.norm()) and exact <= 0.2 * float(target.norm())


def test_streams_and_again():
    """The same bits on another stream, and again; lists of few and of many tensors."""
    for many in (3, 80):
        outs = []
        side = torch.cuda.Stream()
        for stream in (None, side, None):
            tensors = [Tensor((400 + 7 * i,), F32, F16, F16, i % 2 == 0, i) for i in range(many)]
            norm = torch.tensor([3.0], device=DEV)
            side.wait_stream(torch.cuda.current_stream())
            run(tensors, step=4, norm=norm, max_norm=1.0, stream=stream)
            torch.cuda.synchronize()
            outs.append([x for t in tensors for x in (t.p, t.m, t.v, t.copy)])
        for o in outs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(outs[0], o))


@pytest.mark.parametrize("bytes_", [False, True])
@pytest.mark.parametrize("by_row", [False, True])
@pytest.mark.parametrize("k", [3, 16, 1000])
def test_a_small_decay_is_as_large_as_it_should_be(k, by_row, bytes_):
    """lr weight_decay = d = (k + 1/2) 2^-24: exact as a product, and in the middle between two values of 1 - d.  The change d p of parameters in [1, 2) is rounded to
    steps of 2^-23, to either side: what d p / 2^-23, which runs over L = k / 2 + 1 / 4 steps, is off by evens out over whole steps, and leaves an eighth of a step times
    1 / L in the mean at most.  2^20 values of p stand for all of them: their mean is off by 2 L 2^-20 < 2^-10 steps at most (a sawtooth of L teeth).  The product rounds by U."""
    n, d = 1 << 20, (k + 0.5) * 2.0 ** -24
    p = (1 + torch.arange(n, device=DEV) * 2.0 ** -20).reshape(-1, 512 if by_row else n)
    p = p if by_row else p.reshape(-1)
    before = p.clone()
    g, m, v = torch.zeros_like(p), torch.zeros_like(p), torch.zeros_like(p)
    scales = {}
    if bytes_:
        m, v = m.to(torch.int8), v.to(torch.uint8)
        shape = (p.shape[0], 4) if by_row else (n // B,)
        scales = dict(m_scales=[torch.zeros(shape, device=DEV)], v_scales=[torch.zeros(shape, device=DEV)])
    smfg.adamw(smfg.adamw_list([p], [g], [m], [v], weight_decay=(k + 0.5) * 2.0 ** -14, **scales), 1, 2.0 ** -10)
    moved = float((before.double() - p.double()).mean())
    want = d * float(before.double().mean())
    assert abs(moved - want) <= 2.0 ** -23 * (1 / 8 / (k / 2 + 0.25) + 2.0 ** -10) + 2 * U * want
    # and each by its own
    assert float(((before.double() - p.double()) - d * before.double()).abs().max()) <= 2.0 ** -24 * 1.001 + 2 * U * d * 2


@pytest.mark.parametrize("beta2,factor,most", [(0.999, 0.0, 250), (0.999, 2.0, 250), (0.999, 10.0, 60), (0.99, 0.0, 230), (0.95, 0.0, 250), (0.95, 2.0, 128)])
def test_second_moments_of_8_bits_over_many_steps(beta2, factor, most):
    """One element of a block keeps its gradient, all others' have become `factor` times their root of v.  The states are the ones that the definition with its rounding gives,
    step by step in 64 bits, for all whose number is never within 2^-10 of the middle between two (v is off by 23 U, its root's root by a quarter, and by 6 U for itself: below
    2^-12 of up to 255).  A number stays for good where a step changes it by less than a half, and the moment then has its share of the block's largest: the
    deviation from the moments without rounding is what it is by that."""
    steps = 200
    k = torch.ceil(torch.arange(1, B + 1, dtype=torch.float64) * most / B)
    k[0] = 255
    first, g = k.clone(), (factor * (k / 255) ** 2).float()
    g[0] = 1.0
    p, m, v = torch.zeros(B, device=DEV), torch.zeros(B, dtype=torch.int8, device=DEV), k.to(torch.uint8).to(DEV)
    ms, vs = torch.zeros(1, device=DEV), torch.ones(1, device=DEV)
    lst = smfg.adamw_list([p], [g.to(DEV)], [m], [v], [ms], [vs])
    gg, top, exact, apart = g.double(), 1.0, (k / 255) ** 4, torch.ones(B, dtype=torch.float64)
    for i in range(1, steps + 1):
        smfg.adamw(lst, i, LR, betas=(B1, beta2), eps=EPS)
        root = torch.sqrt(beta2 * (top * (k / 255) ** 2) ** 2 + (1 - beta2) * gg * gg)
        exact = beta2 * exact + (1 - beta2) * gg * gg
        top = float(root.max())
        x = 255 * torch.sqrt(root / top)
        apart = torch.minimum(apart, (x % 1 - 0.5).abs())
        k = torch.round(x).clamp(min=1)
    sure = apart > 2.0 ** -10
    assert int(sure.sum()) >= 96
    assert torch.equal(v.cpu()[sure].double(), k[sure])
    # the root of v is off by 15 U a step relative to the block's largest, which has nothing to be rounded to
    assert abs(float(vs) - top) <= 20 * steps * U * top
    still = (first * (1 + (1 - beta2) * (factor ** 2 - 1)) ** 0.25 - first).abs() < 0.499
    still[0] = True
    assert torch.equal(k[still], first[still]) and bool((k != first)[~still].all())
    out = torch.empty(B, device=DEV)
    smfg.adamw_values(v, vs, out)
    share = (top * (k / 255) ** 2) ** 2
    assert bool(((out.cpu().double() - share).abs() <= (2 * 20 * steps + 11) * U * share)[sure].all())
    off = (share / exact)[1:]
    if factor == 0.0:  # what stays is too large by what the moment should have lost
        want = beta2 ** -steps
        assert bool((((off - want).abs() <= 1e-9 * want) == still[1:]).all()) and bool((off <= want * (1 + 1e-9)).all())
    else:  # what stays is too small by what it should have gained
        want = 1 / (beta2 ** steps + (1 - beta2 ** steps) * factor ** 2)
        assert bool((((off - want).abs() <= 1e-6 * want) == still[1:]).all()) and bool((off >= want * (1 - 1e-6)).all())


@pytest.mark.parametrize("bytes_", [False, True])
@pytest.mark.parametrize("ptype", [F32, F16, BF16])
@pytest.mark.parametrize("decay", [0.0, WD])
def test_infinite_parameters_stay_infinite(decay, ptype, bytes_):
    """A parameter of -infinity masks what it is added to; a step with a finite gradient leaves it there, a NaN is one behind the step too, and the others take theirs."""
    t = Tensor((1000,), ptype, ptype, None, bytes_, 11, decay=decay)
    t.p[7::100], t.p[8::100], t.p[9::100] = float("-inf"), float("inf"), float("nan")
    t.g[7:500:100] = 0.0
    before = (t.p.clone(), t.state(), t.g.clone())
    run([t], step=3)
    fine = before[0].isfinite()
    assert int(fine.sum()) == 970 and torch.equal(t.p.isnan(), before[0].isnan()) and bool((t.p[7::100] == float("-inf")).all()) and bool((t.p[8::100] == float("inf")).all())
    want, _, _, tp, _, _ = step_of(*before[:1], *before[1][:2], before[2], *before[1][2:], 3, 1.0, decay)
    check(t.p[fine], want[fine], rounded(tp, want, ptype)[fine])
