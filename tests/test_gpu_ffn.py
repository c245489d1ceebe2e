"""GPU parity of the gated feed-forward block (m3_ffn_fwd, m3_ffn_bwd) against
its definition in fp64 and against central differences of it.

Bars.  u = 2^-24.  A sum of K products accumulated in fp32 is off by at most
(8 + 2 sqrt K) u of the sum of their magnitudes (independent roundings).  In
bf16 the values between the products (h, dg, du) are rounded once, each off by
at most 2^-9 of itself, uniformly: a sum over them by 6 standard deviations,
6 2^-9 / sqrt 3 of the root of the sum of the squared products; and the result
itself is rounded, 2^-8 of it.
"""
import pytest
import torch

from paper_2603_15569_amd import m3

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def activation(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    c = (2 / torch.pi) ** 0.5
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def reference(x, Wg, Wu, Wd, dy=None, act="silu", io=torch.float32):
    """Results in fp64 and their bars, by name."""
    x, Wg, Wu, Wd = (t.detach().double() for t in (x, Wg, Wu, Wd))
    b16 = io == torch.bfloat16
    sums = lambda K: (8 + 2 * K ** 0.5) * U  # noqa: E731
    mid = 6 * 2.0 ** -9 / 3 ** 0.5 if b16 else 0.0
    end = 2.0 ** -8 if b16 else 2 * U
    T, D, F = x.shape[0], x.shape[1], Wg.shape[0]
    g, u = x @ Wg.T, x @ Wu.T
    eg, eu = (sums(D) * (x.abs() @ W.abs().T) for W in (Wg, Wu))
    f, df = activation(g, act)
    h = f * u
    eh = (df.abs() + 4 * U) * eg * u.abs() + f.abs() * eu + 8 * U * h.abs()
    y = h @ Wd.T
    out = dict(y=(y, eh @ Wd.abs().T + sums(F) * (h.abs() @ Wd.abs().T)
                  + mid * ((h ** 2) @ (Wd ** 2).T).sqrt() + end * y.abs()))
    if dy is not None:
        dy = dy.detach().double()
        dh = dy @ Wd
        edh = sums(D) * (dy.abs() @ Wd.abs())
        du, dg = dh * f, dh * u * df
        # (the slopes of act and of act' are below 2 in magnitude)
        edu = edh * f.abs() + 2 * dh.abs() * eg + 8 * U * du.abs()
        edg = edh * (u * df).abs() + dh.abs() * (eu * df.abs() + 2 * u.abs() * eg) + 8 * U * (dh * u).abs() * 2

        def product(a, ea, b):
            v = a.T @ b
            return v, ea.T @ b.abs() + sums(T) * (a.abs().T @ b.abs()) + mid * ((a ** 2).T @ (b ** 2)).sqrt() + end * v.abs()
        dx = dg @ Wg + du @ Wu
        out["dx"] = (dx, edg @ Wg.abs() + edu @ Wu.abs() + sums(2 * F) * (dg.abs() @ Wg.abs() + du.abs() @ Wu.abs())
                     + mid * ((dg ** 2) @ (Wg ** 2) + (du ** 2) @ (Wu ** 2)).sqrt() + end * dx.abs())
        out["dWg"], out["dWu"] = product(dg, edg, x), product(du, edu, x)
        v = dy.T @ h
        out["dWd"] = (v, dy.abs().T @ eh + sums(T) * (dy.abs().T @ h.abs())
                      + mid * ((dy ** 2).T @ (h ** 2)).sqrt() + end * v.abs())
    return out


def inputs(T, D, F, io, seed, layout="plain"):
    g = torch.Generator(DEV).manual_seed(seed)

    def rand(*shape, scale=1.0):
        return (torch.randn(shape, device=DEV, generator=g) * scale).to(io)
    if layout == "packed":       # a slice of a wider row, its neighbours not finite
        x, dy = torch.full((2, T, 3 * D + 2), float("nan"), device=DEV, dtype=io).unbind(0)
        x, dy = x[:, D:2 * D], dy[:, 1:D + 1]
        x.copy_(rand(T, D))
        dy.copy_(rand(T, D))
    elif layout == "head":       # the first rows of a longer array, the rest not finite
        x, dy = torch.full((2, T + 70, D), float("nan"), device=DEV, dtype=io).unbind(0)
        x, dy = x[:T], dy[:T]
        x.copy_(rand(T, D))
        dy.copy_(rand(T, D))
    else:
        x, dy = rand(T, D), rand(T, D)
    return x, rand(F, D, scale=D ** -0.5), rand(F, D, scale=D ** -0.5), rand(D, F, scale=F ** -0.5), dy


def check(name, got, ref):
    v, bar = ref
    err = (got.double() - v).abs()
    assert torch.isfinite(got).all() and (err <= bar).all(), \
        f"{name}: {err.max().item():.3e} off at a largest value of {v.abs().max().item():.3e}, " \
        f"{(err > bar).sum().item()} of {err.numel()} beyond the bar"


SIZES = [(1, 1, 1), (1, 64, 128), (2, 65, 67), (3, 7, 300), (16, 256, 512), (17, 100, 300), (48, 520, 1344),
         (64, 130, 100), (65, 130, 100), (129, 256, 768), (300, 512, 1100), (520, 264, 264), (1030, 72, 40)]


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("act,layout", [("silu", "plain"), ("gelu", "packed"), ("silu", "head")])
def test_forward_and_backward(io, size, act, layout):
    T, D, F = size
    say(f"ffn {size} {io} {act} {layout}")
    x, Wg, Wu, Wd, dy = inputs(T, D, F, io, T + D + F, layout)
    y = m3.ffn_fwd(x, Wg, Wu, Wd, act=act)
    g = m3.ffn_bwd(x, Wg, Wu, Wd, dy, act=act)
    ref = reference(x, Wg, Wu, Wd, dy, act, io)
    for name, got in dict(y=y, **g).items():
        check(name, got, ref[name])


@pytest.mark.parametrize("io,T,D,F", [(torch.bfloat16, 3000, 512, 320), (torch.bfloat16, 700, 1000, 2730),
                                      (torch.float32, 1500, 264, 1032), (torch.bfloat16, 8192, 264, 256)])
def test_tiles_and_splits(io, T, D, F):
    """Sizes that take the larger tiles, and few tiles with a long sum (split)."""
    say(f"ffn {T} {D} {F} {io}")
    x, Wg, Wu, Wd, dy = inputs(T, D, F, io, 3, "plain")
    ref = reference(x, Wg, Wu, Wd, dy, "gelu", io)
    check("y", m3.ffn_fwd(x, Wg, Wu, Wd, act="gelu"), ref["y"])
    for name, got in m3.ffn_bwd(x, Wg, Wu, Wd, dy, act="gelu").items():
        check(name, got, ref[name])


def test_batched_rows_and_given_output():
    x, Wg, Wu, Wd, dy = inputs(30, 96, 160, torch.bfloat16, 5)
    y = m3.ffn_fwd(x, Wg, Wu, Wd)
    out = torch.empty(2, 15, 96, device=DEV, dtype=torch.bfloat16)
    assert m3.ffn_fwd(x.view(2, 15, 96), Wg, Wu, Wd, out=out) is out and torch.equal(out.view(30, 96), y)
    g, gb = m3.ffn_bwd(x, Wg, Wu, Wd, dy), m3.ffn_bwd(x.view(2, 15, 96), Wg, Wu, Wd, dy.view(2, 15, 96))
    assert gb["dx"].shape == (2, 15, 96) and torch.equal(gb["dx"].view(30, 96), g["dx"])
    assert all(torch.equal(g[k], gb[k]) for k in ("dWg", "dWu", "dWd"))


def test_no_tokens():
    _, Wg, Wu, Wd, _ = inputs(1, 40, 56, torch.bfloat16, 5)
    x = torch.zeros(0, 40, device=DEV, dtype=torch.bfloat16)
    assert m3.ffn_fwd(x, Wg, Wu, Wd).shape == (0, 40)
    g = m3.ffn_bwd(x, Wg, Wu, Wd, x)
    assert g["dx"].shape == (0, 40) and all(not g[k].any() and g[k].shape == W.shape
                                            for k, W in (("dWg", Wg), ("dWu", Wu), ("dWd", Wd)))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_against_differences(act):
    """The kernel's gradient along a direction against central differences of the
    definition in fp64 (step 1e-5: their own error is below 1e-8)."""
    x, Wg, Wu, Wd, dy = inputs(70, 24, 40, torch.float32, 8)
    g = m3.ffn_bwd(x, Wg, Wu, Wd, dy, act=act)
    host = dict(x=x, Wg=Wg, Wu=Wu, Wd=Wd)
    host = {k: v.double() for k, v in host.items()}

    def J(**over):
        a = {**host, **over}
        return (reference(a["x"], a["Wg"], a["Wu"], a["Wd"], act=act)["y"][0] * dy.double()).sum().item()
    gen = torch.Generator(DEV).manual_seed(2)
    for name in host:
        d = torch.randn(host[name].shape, generator=gen, dtype=torch.float64, device=DEV)
        want = (J(**{name: host[name] + 1e-5 * d}) - J(**{name: host[name] - 1e-5 * d})) / 2e-5
        have = (g["d" + name].double() * d).sum().item()
        assert abs(have - want) <= 1e-5 * (g["d" + name].double() * d).abs().sum().item() + 1e-6, name


@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_nonfinite_rows_stay_theirs(T, io):
    """A token that is not finite spoils its own row of y, no other; large gates
    saturate without NaN."""
    x, Wg, Wu, Wd, _ = inputs(T, 72, 136, io, 4)
    clean = m3.ffn_fwd(x, Wg, Wu, Wd)
    x[3, 5], x[1, 70] = float("nan"), float("inf")
    y = m3.ffn_fwd(x, Wg, Wu, Wd)
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[3] = keep[1] = False
    assert torch.equal(y[keep], clean[keep]) and not torch.isfinite(y[~keep]).any()
    for act in ("silu", "gelu"):
        big = torch.full((T, 72), 1e4, device=DEV, dtype=io)
        big[::2] *= -1
        one = torch.ones_like(Wg)
        y = m3.ffn_fwd(big, one, one, Wd * 0 + 1e-8, act=act)
        assert torch.isfinite(y).all() and not y[::2].any()
        g = m3.ffn_bwd(big, one, one, Wd * 0 + 1e-8, big * 0 + 1, act=act)
        assert all(torch.isfinite(v).all() for v in g.values())


def test_same_bits_on_every_run_and_stream():
    for T in (7, 300):
        x, Wg, Wu, Wd, dy = inputs(T, 256, 704, torch.bfloat16, 6)
        ws = m3.ffn_workspace(x, Wg, backward=True)
        both = lambda: [m3.ffn_fwd(x, Wg, Wu, Wd, workspace=ws),  # noqa: E731
                        *m3.ffn_bwd(x, Wg, Wu, Wd, dy, workspace=ws).values()]
        ref = both()
        side = torch.cuda.Stream()
        for _ in range(3):
            ws.fill_(255)      # (the workspace needs no initialisation: all NaN)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                got = both()
            torch.cuda.current_stream().wait_stream(side)
            assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_captured_and_replayed():
    x, Wg, Wu, Wd, dy = inputs(100, 256, 704, torch.bfloat16, 6)
    ws = m3.ffn_workspace(x, Wg, backward=True)
    both = lambda: [m3.ffn_fwd(x[:9], Wg, Wu, Wd, workspace=ws),  # noqa: E731
                    *m3.ffn_bwd(x, Wg, Wu, Wd, dy, workspace=ws).values()]
    ref = both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(4):
        for o in out:
            o.fill_(3.0)
        eager = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(ref, out, eager))


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 264, 8260), (9, 40, 12300), (33, 264, 8260), (64, 264, 8260), (50, 2056, 1000),
                                  (17, 4100, 24)], ids=str)
def test_few_tokens_of_wide_weights(io, size):
    """Workgroups of up to 48 rows of weights, the last of a few, k in parts."""
    T, D, F = size
    say(f"ffn few {size} {io}")
    x, Wg, Wu, Wd, _ = inputs(T, D, F, io, seed=T + F)
    check("y", m3.ffn_fwd(x, Wg, Wu, Wd), reference(x, Wg, Wu, Wd, io=io)["y"])


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_backward_in_runs_of_tokens(io):
    """So wide that dh is formed for 256 tokens at a time.  Half a million sums an
    output: the values between the products are followed through their rounding
    one by one.  With e the fp32 error of v, the stored value lies between v - e
    and v + e rounded; what that leaves open, the sums' own errors and the
    result's rounding (2^-8 of it in bf16) make the bar."""
    say(f"ffn runs {io}")
    T, D, F = 600, 16, 32900
    x, Wg, Wu, Wd, dy = inputs(T, D, F, io, seed=5)
    got = m3.ffn_bwd(x, Wg, Wu, Wd, dy)
    x, Wg, Wu, Wd, dy = (t.double() for t in (x, Wg, Wu, Wd, dy))
    sums = lambda K: (8 + 2 * K ** 0.5) * U  # noqa: E731
    end = 2.0 ** -8 if io == torch.bfloat16 else 2 * U
    g, u, dh = x @ Wg.T, x @ Wu.T, dy @ Wd
    eg, eu, edh = (sums(D) * e for e in (x.abs() @ Wg.abs().T, x.abs() @ Wu.abs().T, dy.abs() @ Wd.abs()))
    f, df = activation(g, "silu")

    def stored(v, e):
        r, lo, hi = (w.to(io).double() for w in (v, v - e, v + e))
        return r, torch.maximum(hi - r, r - lo)
    h, eh = stored(f * u, (df.abs() + 4 * U) * eg * u.abs() + f.abs() * eu + 8 * U * (f * u).abs())
    du, edu = stored(dh * f, edh * f.abs() + 2 * dh.abs() * eg + 8 * U * (dh * f).abs())
    dg, edg = stored(dh * u * df, edh * (u * df).abs() + dh.abs() * (eu * df.abs() + 2 * u.abs() * eg)
                     + 16 * U * (dh * u).abs())

    def bar(v, e, K, size):
        return v, e + sums(K) * size + end * v.abs()
    check("dx", got["dx"], bar(dg @ Wg + du @ Wu, edg @ Wg.abs() + edu @ Wu.abs(), 2 * F,
                               dg.abs() @ Wg.abs() + du.abs() @ Wu.abs()))
    for name, a, e, b in (("dWg", dg, edg, x), ("dWu", du, edu, x), ("dWd", h, eh, dy)):
        v, err, size = a.T @ b, e.T @ b.abs(), a.abs().T @ b.abs()
        if name == "dWd":
            v, err, size = v.T, err.T, size.T
        check(name, got[name], bar(v, err, T, size))


def test_more_rows_to_copy_than_workgroups():
    """Rows of an odd width, copied: more of them than the copy has workgroups."""
    say("ffn 70001 rows of 3")
    x, Wg, Wu, Wd, dy = inputs(70001, 3, 5, torch.float32, 9)
    y, ref = m3.ffn_fwd(x, Wg, Wu, Wd), reference(x, Wg, Wu, Wd, dy)
    check("y", y, ref["y"])
    for name, got in m3.ffn_bwd(x, Wg, Wu, Wd, dy).items():
        check(name, got, ref[name])


def test_given_stream_without_a_workspace():
    """`stream` as an argument: workspace and outputs are in that stream's order."""
    x, Wg, Wu, Wd, dy = inputs(300, 256, 704, torch.bfloat16, 6)
    both = lambda **kw: [m3.ffn_fwd(x, Wg, Wu, Wd, **kw), *m3.ffn_bwd(x, Wg, Wu, Wd, dy, **kw).values()]  # noqa: E731
    ref = both()
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    side.wait_stream(here)
    for _ in range(3):
        got = both(stream=side)
        busy = torch.full((64 << 20,), 171, dtype=torch.uint8, device=DEV)   # (memory that a call gave back too early)
        here.wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(ref, got))
        del busy


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,D,F", [(1, 64, 128), (9, 72, 40), (100, 128, 264), (300, 64, 100)])
def test_weights_of_any_start(io, T, D, F):
    """Weights as views that start on any element of a buffer, with the workspace left to
    the call, or kept with room for them; without room they are refused."""
    say(f"ffn any start {T} {D} {F} {io}")
    x, Wg, Wu, Wd, dy = inputs(T, D, F, io, 31)
    ref = reference(x, Wg, Wu, Wd, dy, "gelu", io)
    buf = torch.full((3 * D * F + 30,), float("nan"), device=DEV, dtype=io)
    views = []
    for k, W in enumerate((Wg, Wu, Wd)):
        at = k * (D * F + 9) + 1
        views.append(buf[at:at + D * F].view(W.shape).copy_(W))
    assert any(v.data_ptr() % 16 for v in views)
    for weights in (views, [views[0], Wu, Wd], [Wg, Wu, views[2]]):
        if not any(v.data_ptr() % 16 for v in weights):
            continue
        ws = m3.ffn_workspace(x, Wg, backward=True, any_weights=True)
        for kw in ({}, dict(workspace=ws)):
            check("y", m3.ffn_fwd(x, *weights, act="gelu", **kw), ref["y"])
            for name, got in m3.ffn_bwd(x, *weights, dy, act="gelu", **kw).items():
                check(name, got, ref[name])
    es = 4 if io == torch.float32 else 2
    if D * es % 16 == 0 and views[0].data_ptr() % 16:
        with pytest.raises(m3.M3Error):
            m3.ffn_fwd(x, *views, workspace=m3.ffn_workspace(x, Wg))
