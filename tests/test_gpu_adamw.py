"""GPU parity of the AdamW step over many tensors (m3_adamw_step) against its
formula in fp64.

Bars.  u = 2^-24.  m and v are three roundings from the formula on the same
states (m's of its terms, which may cancel); p is its own rounding, the
update's, whose root, quotient and products are ten, and m's through it.  8-bit states are held to the scale of their block exactly as
the formula's largest magnitude gives it, and each to one step of e4m3 around
the moving average it stands for.
"""
import pytest
import torch

from paper_2603_15569_amd import m3

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
BLOCK = 256
SHAPES = [(1,), (3, 5), (255,), (256,), (257,), (33, 31), (0,), (1000,), (1024,), (1025,), (4, 700), (20011,)]


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)


class Case:
    """Tensors carved out of one buffer each, at odd places, with guards between."""

    def __init__(self, seed, eight=False, gtype=torch.float32, low=True, shapes=SHAPES, zero=False):
        g = torch.Generator(DEV).manual_seed(seed)
        gap = 5
        sizes = [torch.Size(s).numel() for s in shapes]
        total = sum(sizes) + gap * (len(sizes) + 1)
        at, self.spans = gap, []
        for n in sizes:
            self.spans.append((at, n))
            at += n + gap
        self.shapes, self.eight, self.seed = shapes, eight, seed

        def flat(dtype, scale):
            return (torch.randn(total, device=DEV, generator=g) * scale).to(dtype)
        self.flat = dict(p=flat(torch.float32, 0.02), g=flat(gtype, 1e-3))
        if eight:
            self.flat["m"] = torch.zeros(total, device=DEV, dtype=torch.float8_e4m3fn)
            self.flat["v"] = torch.zeros(total, device=DEV, dtype=torch.float8_e4m3fn)
            self.scales = [torch.zeros(-(-n // BLOCK), 2, device=DEV) for n in sizes]
            if not zero:   # codes and scales of a run under way
                for k in "mv":
                    self.flat[k].copy_((torch.randn(total, device=DEV, generator=g) * 60).clamp(-448, 448)
                                       .abs_() if k == "v" else (torch.randn(total, device=DEV, generator=g) * 60).clamp(-448, 448))
                for s in self.scales:
                    s.copy_(torch.rand(s.shape, device=DEV, generator=g) * 1e-5 + 1e-6)
        else:
            self.flat["m"] = flat(torch.float32, 0.0 if zero else 3e-4)
            self.flat["v"] = flat(torch.float32, 0.0 if zero else 4e-4).square_()
            self.scales = None
        if low:
            self.flat["low"] = torch.full((total,), 7.0, device=DEV, dtype=torch.bfloat16)
        self.decay = [0.1 if len(s) > 1 else 0.0 for s in shapes]
        self.table = m3.adamw_table(self.views("p"), self.views("g"), self.views("m"), self.views("v"),
                                    weight_decay=self.decay, low=self.views("low") if low else None, scales=self.scales)

    def views(self, k):
        return [self.flat[k][a:a + n].view(s) for (a, n), s in zip(self.spans, self.shapes)]

    def state(self, k, which):
        """State k of a tensor in fp64: m, or v."""
        t = self.views(which)[k].double().view(-1)
        if self.eight:
            t = t * self.scales[k][:, "mv".index(which)].double().repeat_interleave(BLOCK)[:t.numel()]
            t = t if which == "m" else t * t
        return t

    def guards(self, k):
        keep = torch.ones_like(self.flat[k], dtype=torch.bool)
        for a, n in self.spans:
            keep[a:a + n] = False
        return self.flat[k][keep].clone()


KW = dict(lr=3e-4, betas=(0.9, 0.95), eps=1e-8)


def expected(c, k, step, scale):
    b1, b2 = KW["betas"]
    g = c.views("g")[k].double().view(-1) * scale
    m = b1 * c.state(k, "m") + (1 - b1) * g
    v = b2 * c.state(k, "v") + (1 - b2) * g * g
    p = c.views("p")[k].double().view(-1)
    slope = KW["lr"] / (1 - b1 ** step) / ((v / (1 - b2 ** step)).sqrt() + KW["eps"])
    upd = slope * m
    bar = 2 * U * p.abs() + 24 * U * upd.abs() + 4 * U * (m.abs() + 1e-3 * 0.1) * slope
    return m, v, p * (1 - KW["lr"] * c.decay[k]) - upd, bar


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16], ids=["gf32", "gbf16"])
@pytest.mark.parametrize("low,scaled,step,zero", [(True, True, 1000, False), (False, False, 1, True)])
def test_step(eight, gtype, low, scaled, step, zero):
    say(f"adamw eight={eight} {gtype} low={low} scaled={scaled} step={step}")
    c = Case(3, eight, gtype, low, zero=zero)
    gs = torch.full((1,), 0.37, device=DEV) if scaled else None
    scale = gs.double().item() if scaled else 1.0
    want = [expected(c, k, step, scale) for k in range(len(SHAPES))]
    guards = {k: c.guards(k) for k in c.flat}
    m3.adamw_step(c.table, step=step, seed=99, grad_scale=gs, **KW)
    for k, (m, v, p, bar) in enumerate(want):
        if p.numel() == 0:
            continue
        # the formula's terms: two products and a sum each, on states known to fp32
        for name, ref, got in (("m", m, c.views("m")[k]), ("v", v, c.views("v")[k])):
            if not eight:
                big = ref.abs() + (1e-3 * 0.1 if name == "m" else 0)
                assert ((got.double().view(-1) - ref).abs() <= 4 * U * big).all(), (k, name)
                continue
            col = "mv".index(name)
            root = ref if name == "m" else ref.sqrt()
            rows = torch.nn.functional.pad(root, (0, -root.numel() % BLOCK)).view(-1, BLOCK)
            most = rows.abs().amax(1)
            sc = c.scales[k][:, col].double()
            assert ((sc - most / 448).abs() <= 8 * U * most / 448).all(), (k, name)
            by = sc.repeat_interleave(BLOCK)[:root.numel()]
            code = got.double().view(-1)
            # one step of e4m3 where the number lies: 2^-3 of its power of two, 2^-9 below 2^-6
            x = torch.where(by > 0, root / by, 0.0)
            quantum = 2.0 ** (torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
            assert ((code - x).abs() <= quantum * (1 + 1e-4)).all(), (k, name)
            if name == "v":
                assert ((code > 0) == (root > 0)).all()
        assert ((c.views("p")[k].double().view(-1) - p).abs() <= bar).all(), k
        if low:
            assert torch.equal(c.views("low")[k], c.views("p")[k].to(torch.bfloat16))
    for k, before in guards.items():
        assert torch.equal(c.guards(k).view(torch.uint8), before.view(torch.uint8)), k


def test_eight_bits_follow_the_average_without_bias():
    """The codes' rounding is zero on average: over 200000 elements the mean error in
    units of a step is within five standard deviations of none (a rounding to
    nearest or down is not: its mean error depends on where the numbers lie)."""
    shapes = [(200000,)]
    c = Case(5, True, shapes=shapes, low=False, zero=True)
    c.flat["g"].copy_(torch.rand(c.flat["g"].shape, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) + 0.5)
    m, v, _, _ = expected(c, 0, 1, 1.0)
    m3.adamw_step(c.table, step=1, seed=3, **KW)
    for name, ref in (("m", m), ("v", v.sqrt())):
        by = c.scales[0][:, "mv".index(name)].double().repeat_interleave(BLOCK)[:ref.numel()]
        x = ref / by
        quantum = 2.0 ** (torch.floor(torch.log2(x)) - 3)
        e = (c.views(name)[0].double() - x) / quantum
        free = x < 440      # (the block's largest are stored exactly)
        assert e[free].abs().max() <= 1.0 + 1e-6
        sd = e[free].std().item() / free.sum().item() ** 0.5
        assert abs(e[free].mean().item()) <= 5 * sd, (name, e[free].mean().item(), sd)


def test_eight_bits_move_a_slow_average():
    """Steps too small for a rounding to nearest to move the state still move it: after
    200 steps of a gradient half as large as the state, v is near the average's value."""
    n = 64 * BLOCK
    c = Case(6, True, shapes=[(n,)], low=False, zero=True)
    g = c.flat["g"]
    g.fill_(1.0)
    kw = dict(lr=0.0, betas=(0.9, 0.99), eps=1e-8)
    m3.adamw_step(c.table, step=1, seed=0, **kw)          # v = 0.01 everywhere
    half = torch.zeros_like(g)
    half[c.spans[0][0]:c.spans[0][0] + n:2] = 1.0          # every second element's gradient stays at 0.1
    g.copy_(0.1 * half + 0.2 * (1 - half))
    ref = torch.full((n,), 0.01, dtype=torch.float64, device=DEV)
    for t in range(2, 202):
        m3.adamw_step(c.table, step=t, seed=t, **kw)
        ref = 0.99 * ref + 0.01 * c.views("g")[0].double() ** 2
    got = c.state(0, "v")
    for part in (slice(0, None, 2), slice(1, None, 2)):
        assert abs(got[part].mean().item() / ref[part].mean().item() - 1) < 0.05


def test_seeds_and_repeats():
    runs = []
    for seed in (1, 1, 2):
        c = Case(7, True)
        for t in range(1, 4):
            m3.adamw_step(c.table, step=t, seed=seed * 10 + t, **KW)
        runs.append([c.flat[k].view(torch.uint8).clone() for k in ("p", "m", "v", "low")] + [s.clone() for s in c.scales])
    assert all(torch.equal(a, b) for a, b in zip(runs[0], runs[1]))
    assert not torch.equal(runs[0][1], runs[2][1])


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
def test_nonfinite_and_zero_gradients(eight):
    """A gradient that is not finite spoils its element, or its block of 256 in 8 bits,
    and nothing else; zero gradients of a zero state change p by the decay alone."""
    def run(poison):
        c = Case(8, eight, shapes=[(700,), (40, 30)], low=False)
        if poison is not None:
            c.views("g")[0][300] = poison
        m3.adamw_step(c.table, step=5, seed=4, **KW)
        m3.adamw_step(c.table, step=6, seed=5, **KW)
        return c
    clean = run(None)
    for poison in (float("nan"), float("inf")):
        c = run(poison)
        keep = torch.ones(700, dtype=torch.bool, device=DEV)
        keep[256:512] = False
        if not eight:
            keep[:] = True
            keep[300] = False
        assert torch.equal(c.views("p")[0][keep], clean.views("p")[0][keep])
        assert torch.equal(c.views("p")[1], clean.views("p")[1])
        assert not torch.isfinite(c.views("p")[0][300])
    c = Case(9, eight, shapes=[(30, 40)], low=False, zero=True)
    c.flat["g"].zero_()
    before = c.views("p")[0].double()
    m3.adamw_step(c.table, step=1, seed=4, **KW)
    assert ((c.views("p")[0].double() - before * (1 - KW["lr"] * 0.1)).abs() <= 2 * U * before.abs()).all()
    assert not c.views("m")[0].float().any() and not c.views("v")[0].float().any()


def test_many_tensors_on_a_side_stream_and_captured():
    shapes = [(1 + 37 * k % 900,) for k in range(300)]
    a, b = Case(10, shapes=shapes), Case(10, shapes=shapes)
    m3.adamw_step(a.table, step=1, **KW)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m3.adamw_step(b.table, step=1, **KW)
    torch.cuda.current_stream().wait_stream(side)
    same = lambda: all(torch.equal(a.flat[k], b.flat[k]) for k in a.flat)  # noqa: E731
    assert same()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m3.adamw_step(b.table, step=2, **KW)
    for _ in range(3):
        m3.adamw_step(a.table, step=2, **KW)
        graph.replay()
        torch.cuda.synchronize()
        assert same()


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16], ids=["gf32", "gbf16"])
def test_small_gradients_without_eps(eight, gtype):
    """Gradients of 1e-17 to 3e-21 on a zero state with eps = 0: v goes below the smallest
    normal number, and the step is still the formula's, about lr.  A subnormal v is
    known to three halves of 2^-149 (its square, its product and its sum), the step to
    half of what that is of v; the rest as for every step."""
    say(f"adamw small gradients eight={eight} {gtype}")
    c = Case(11, eight, gtype, low=False, shapes=[(300,), (1025,)], zero=True)
    total = c.flat["g"].numel()
    gen = torch.Generator(DEV).manual_seed(4)
    size = 10.0 ** (-17 - 3.5 * torch.rand(total, device=DEV, generator=gen, dtype=torch.float64))
    sign = torch.randint(0, 2, (total,), device=DEV, generator=gen) * 2 - 1
    c.flat["g"].copy_((size * sign).to(gtype))
    lr, (b1, b2) = KW["lr"], KW["betas"]
    want = []
    for k in range(2):
        g, p = c.views("g")[k].double(), c.views("p")[k].double()
        v = (1 - b2) * g * g
        upd = lr * g / g.abs()
        off = 1.5 * 2.0 ** -149 / v
        want.append((p - upd, 2 * U * p.abs() + upd.abs() * (28 * U + off), v.sqrt(), off))
    m3.adamw_step(c.table, step=1, lr=lr, betas=(b1, b2), eps=0.0, seed=5)
    for k, (p, bar, rv, off) in enumerate(want):
        got = c.views("p")[k]
        assert torch.isfinite(got).all() and ((got.double() - p).abs() <= bar).all(), k
        if eight:
            rows = torch.nn.functional.pad(rv, (0, -rv.numel() % BLOCK)).view(-1, BLOCK)
            at = rows.argmax(1, keepdim=True)
            most = rows.gather(1, at)[:, 0]
            off = torch.nn.functional.pad(off, (0, -off.numel() % BLOCK)).view(-1, BLOCK).gather(1, at)[:, 0]
            assert ((c.scales[k][:, 1].double() - most / 448).abs() <= (8 * U + off) * most / 448).all(), k
            assert c.views("v")[k].float().gt(0).all()
        else:
            assert ((c.views("v")[k].double() - rv ** 2).abs() <= 4 * U * rv ** 2 + 1.5 * 2.0 ** -149).all(), k


@pytest.mark.parametrize("eight", [False, True], ids=["f32", "8bit"])
def test_captured_steps_go_on(eight):
    """A step captured once with t and lr on the device: each replay is the next step,
    with its bias corrections, its lr and its rounding, bit for bit the eager one."""
    a, b = Case(12, eight, shapes=[(700,), (40, 30)]), Case(12, eight, shapes=[(700,), (40, 30)])
    t = torch.ones(1, dtype=torch.int64, device=DEV)
    lr = torch.full((1,), 0.5, dtype=torch.float64, device=DEV)
    kw = dict(betas=(0.9, 0.95), eps=1e-8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m3.adamw_step(b.table, step=t, lr=lr, seed=1000, **kw)
        t.add_(1)
    for k in range(1, 6):
        rate = 1e-3 / k
        lr.fill_(rate)
        m3.adamw_step(a.table, step=k, lr=rate, seed=1000 + k, **kw)
        graph.replay()
        torch.cuda.synchronize()
        assert t.item() == k + 1
        for name in a.flat:
            assert torch.equal(a.flat[name].view(torch.uint8), b.flat[name].view(torch.uint8)), (k, name)
        if eight:
            assert all(torch.equal(x, y) for x, y in zip(a.scales, b.scales))
    # not captured, with only one of the two on the device, and a t of no step
    m3.adamw_step(a.table, step=6, lr=1e-4, seed=1006, **kw)
    m3.adamw_step(b.table, step=t, lr=1e-4, seed=1000, **kw)
    m3.adamw_step(a.table, step=7, lr=1e-3 / 5, seed=3, **kw)
    m3.adamw_step(b.table, step=7, lr=lr, seed=3, **kw)
    assert all(torch.equal(a.flat[name].view(torch.uint8), b.flat[name].view(torch.uint8)) for name in a.flat)
    m3.adamw_step(a.table, step=8, lr=1e-4, seed=3, **kw)
    m3.adamw_step(b.table, step=torch.tensor(8), lr=torch.tensor(1e-4, dtype=torch.float64), seed=3, **kw)   # (the host's)
    assert all(torch.equal(a.flat[name].view(torch.uint8), b.flat[name].view(torch.uint8)) for name in a.flat)
    for bad in (dict(step=t.int(), lr=1e-4), dict(step=t.repeat(2), lr=1e-4), dict(step=8, lr=lr.float())):
        with pytest.raises(ValueError):
            m3.adamw_step(b.table, **bad, **kw)
    t.zero_()
    m3.adamw_step(b.table, step=t, lr=1e-4, **kw)
    assert all(torch.isnan(p).all() for p in b.views("p"))
