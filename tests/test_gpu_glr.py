"""GPU parity of the gated linear recurrence (m3_glr_fwd, m3_glr_bwd,
m3_glr_step) against its definition in fp64, token by token, with gradients
by autograd of that loop and by central differences of it.

Bars.  u = 2^-24 is fp32's rounding.  A token's decay and input carry a few
roundings (elementary functions of one or two ulps among them) and the state
sums the tokens' independent ones, so fp32 results are held to 16 u (1 +
sqrt(L)) of the tensor's largest magnitude (dA: of the sum of its terms'
magnitudes).  bf16 results add their one rounding, 2^-8 of the element.
"""
import numpy as np
import pytest
import torch

from paper_2603_15569_amd import m3

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def reference(x, r, i, A, z=None, h0=None, dy=None, dfinal=None):
    """y, the final state and, with dy, the gradients; all fp64 on the CPU."""
    t = {k: v.detach().double().cpu().requires_grad_(dy is not None)
         for k, v in dict(x=x, r=r, i=i, A=A, z=z, h0=h0).items() if v is not None}
    B, L, D = x.shape
    h = t.get("h0", torch.zeros(B, D, dtype=torch.float64))
    terms, ys = [], []
    for k in range(L):
        la = t["A"] * torch.sigmoid(t["r"][:, k])
        if dy is not None:
            la.retain_grad()
            terms.append((la, torch.sigmoid(t["r"][:, k]).detach()))
        h = torch.exp(la) * h + torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(t["i"][:, k]) * t["x"][:, k]
        ys.append(h * torch.nn.functional.silu(t["z"][:, k]) if z is not None else h)
    y = torch.stack(ys, 1) if L else torch.zeros(B, 0, D, dtype=torch.float64)
    out = dict(y=y.detach(), final=h.detach())
    if dy is not None:
        J = (y * dy.double().cpu()).sum() + (h * dfinal.double().cpu()).sum()
        J.backward()
        out.update({"d" + k: v.grad for k, v in t.items()})
        out["dinit"] = out.pop("dh0", None)
        out["A_terms"] = sum((g.grad * rho).abs().sum(0) for g, rho in terms)
    return out


def inputs(B, L, D, io, gate, seed, layout="plain", init=True):
    g = torch.Generator(DEV).manual_seed(seed)
    n = 4 if gate else 3

    def rand(*shape, io=torch.float32):
        return torch.randn(shape, device=DEV, generator=g).to(io)
    if layout == "packed":        # slices of one projection's output
        parts = list(rand(B, L, n * D, io=io).split(D, dim=-1))
    elif layout == "time":        # tokens outermost
        parts = [rand(L, B, D, io=io).transpose(0, 1) for _ in range(n)]
    elif layout == "odd":         # odd strides and starts
        parts = [rand(B, L, D + 3, io=io)[:, :, 1:D + 1] for _ in range(n)]
    else:
        parts = [rand(B, L, D, io=io) for _ in range(n)]
    A = -torch.exp(np.log(0.0066) + torch.rand((D,), device=DEV, generator=g) * np.log(150.0))
    s = dict(x=parts[0], r=parts[1], i=parts[2], A=A, z=parts[3] if gate else None,
             h0=rand(B, D) if init else None, dy=rand(B, L, D, io=io), dfinal=rand(B, D))
    return s


def close(name, got, ref, L, scale=None):
    got, ref = got.double().cpu(), ref.double()
    tol = 16 * U * (1 + L ** 0.5) * (ref.abs().max() if scale is None else scale)
    if name not in ("final", "dA", "dinit", "state") and close.io == torch.bfloat16:
        tol = tol + 2.0 ** -8 * ref.abs()
    bad = (got - ref).abs() - tol
    assert torch.isfinite(got).all() and (bad <= 0).all(), \
        f"{name}: {((got - ref).abs().max()).item():.3e} off, {(bad > 0).sum().item()} beyond the bar"


SIZES = [(1, 1, 1), (2, 5, 7), (1, 127, 64), (3, 128, 66), (2, 129, 130), (1, 1000, 33),
         (2, 4225, 16), (1, 6000, 2)]   # 34 and 47 tiles: past the reach of one look-back


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("gate,layout,init", [(False, "plain", False), (True, "packed", True),
                                              (True, "odd", False), (False, "time", True)])
def test_forward_and_backward(io, size, gate, layout, init):
    B, L, D = size
    say(f"glr {size} {io} gate={gate} {layout} init={init}")
    s = inputs(B, L, D, io, gate, 11 + L + D, layout, init)
    close.io = io
    ws = m3.glr_workspace(s["x"], s["r"], s["i"], z=s["z"])
    y, fs, st = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], z=s["z"], init_state=s["h0"],
                           save_states=True, workspace=ws)
    g = m3.glr_bwd(s["x"], s["r"], s["i"], s["A"], st, s["dy"], z=s["z"], dfinal=s["dfinal"],
                   want_dinit=init, workspace=ws)
    assert m3.glr_check(s["x"], s["r"], s["i"], ws, z=s["z"]) == 0
    ref = reference(**s)
    close("y", y, ref["y"], L)
    close("final", fs, ref["final"], L)
    for k in ("dx", "dr", "di"):
        close(k, g[k], ref[k], L)
    close("dA", g["dA"], ref["dA"], L, scale=ref["A_terms"])
    if gate:
        close("dz", g["dz"], ref["dz"], L)
    if init:
        close("dinit", g["dinit"], ref["dinit"], L)


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,D,gate", [(1, 1, False), (3, 37, True), (5, 64, False), (70, 130, True)])
def test_step_continues_the_sequence(io, B, D, gate):
    """Steps from the forward's final state are the longer sequence's tokens."""
    say(f"glr step {B} {D} {io} gate={gate}")
    L, more = 20, 5
    s = inputs(B, L + more, D, io, gate, 5 + D)
    close.io = io
    part = lambda t, a, b: None if t is None else t[:, a:b]  # noqa: E731
    _, state = m3.glr_fwd(*(part(s[k], 0, L) for k in ("x", "r", "i")), s["A"], z=part(s["z"], 0, L),
                          init_state=s["h0"])
    ys = [m3.glr_step(state, *(s[k][:, t] for k in ("x", "r", "i")), s["A"],
                      z=None if s["z"] is None else s["z"][:, t]) for t in range(L, L + more)]
    ref = reference(s["x"], s["r"], s["i"], s["A"], s["z"], s["h0"])
    close("y", torch.stack(ys, 1), ref["y"][:, L:], L + more)
    close("state", state, ref["final"], L + more)


def test_continued_prefill_matches_one_call():
    s = inputs(2, 700, 48, torch.float32, True, 3)
    close.io = torch.float32
    args = lambda a, b: [s[k][:, a:b] for k in ("x", "r", "i")]  # noqa: E731
    y1, h = m3.glr_fwd(*args(0, 333), s["A"], z=s["z"][:, :333], init_state=s["h0"])
    y2, h = m3.glr_fwd(*args(333, 700), s["A"], z=s["z"][:, 333:], init_state=h)
    ref = reference(s["x"], s["r"], s["i"], s["A"], s["z"], s["h0"])
    close("y", torch.cat((y1, y2), 1), ref["y"], 700)
    close("final", h, ref["final"], 700)


def test_gradients_against_differences():
    """The kernel's gradient along a direction against central differences of
    the definition in fp64 (step 1e-5: their own error is below 1e-8)."""
    s = inputs(2, 150, 24, torch.float32, True, 9)
    y, fs, st = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], z=s["z"], init_state=s["h0"], save_states=True)
    g = m3.glr_bwd(s["x"], s["r"], s["i"], s["A"], st, s["dy"], z=s["z"], dfinal=s["dfinal"], want_dinit=True)
    host = {k: v.double().cpu() for k, v in s.items()}

    def J(**over):
        a = {**host, **over}
        o = reference(a["x"], a["r"], a["i"], a["A"], a["z"], a["h0"])
        return ((o["y"] * a["dy"]).sum() + (o["final"] * a["dfinal"]).sum()).item()
    gen = torch.Generator().manual_seed(1)
    for name, key in (("x", "dx"), ("r", "dr"), ("i", "di"), ("z", "dz"), ("A", "dA"), ("h0", "dinit")):
        d = torch.randn(host[name].shape, generator=gen, dtype=torch.float64)
        if name == "A":
            d = d * host["A"]      # (a relative change: A stays negative)
        e = 1e-5
        want = (J(**{name: host[name] + e * d}) - J(**{name: host[name] - e * d})) / (2 * e)
        have = (g[key].double().cpu() * d).sum().item()
        size = (g[key].double().cpu() * d).abs().sum().item()
        assert abs(have - want) <= 1e-5 * size + 1e-6, (name, have, want)


def test_lengths_of_zero_and_one_token():
    for io in (torch.bfloat16, torch.float32):
        x = torch.zeros(2, 0, 6, dtype=io, device=DEV)
        A, h0 = -torch.ones(6, device=DEV), torch.randn(2, 6, device=DEV)
        y, fs, st = m3.glr_fwd(x, x, x, A, init_state=h0, save_states=True)
        assert y.shape == (2, 0, 6) and torch.equal(fs, h0) and st.shape == (2, 0, 6)
        assert torch.equal(m3.glr_fwd(x, x, x, A)[1], torch.zeros_like(h0))
        g = m3.glr_bwd(x, x, x, A, st, x, dfinal=h0, want_dinit=True)
        assert torch.equal(g["dinit"], h0) and torch.equal(g["dA"], torch.zeros_like(A))


def test_closed_gates_and_resets():
    """r so low that a = 1: the state is kept, the input has no weight, gradients are
    finite; A so low that an open gate forgets: the state is the token's input."""
    B, L, D = 1, 300, 8
    s = inputs(B, L, D, torch.float32, False, 4)
    s["r"][:, 100:200] = -200.0
    s["r"][:, 250] = float("-inf")
    y, fs, st = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], init_state=s["h0"], save_states=True)
    # (a token's state is formed from the state entering its run: a rounding apart)
    assert ((y[:, 100:200] - y[:, 99:100]).abs() <= 8 * U * y.abs().max()).all()
    assert ((y[:, 250] - y[:, 249]).abs() <= 8 * U * y.abs().max()).all()
    g = m3.glr_bwd(s["x"], s["r"], s["i"], s["A"], st, s["dy"], dfinal=s["dfinal"])
    assert all(torch.isfinite(v).all() for v in g.values())
    assert torch.equal(g["dr"][:, 100:200], torch.zeros_like(g["dr"][:, 100:200]))
    A = torch.full((D,), -1e30, device=DEV)
    y, _ = m3.glr_fwd(s["x"], torch.zeros_like(s["r"]), s["i"], A)
    ref = torch.sigmoid(s["i"].double()) * s["x"].double()
    assert ((y.double() - ref).abs() <= 8 * U * ref.abs()).all()


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("gate", [False, True])
def test_nearly_closed_gates(io, gate):
    """r from -82 to -90, where 1 - a^2 goes below the smallest normal number before
    rho is zero: everything is finite and as the definition gives it."""
    say(f"glr nearly closed {io} gate={gate}")
    decays = [0.005, 0.0066, 0.02, 0.05, 0.1, 0.3, 0.5, 1.0]
    B, L, D = 2, 200, len(decays)
    s = inputs(B, L, D, io, gate, 21)
    s["A"] = -torch.tensor(decays, device=DEV)
    s["r"][:, 60:125] = torch.linspace(-82.0, -90.0, 65, device=DEV).to(io)[:, None]
    s["r"][:, 150] = -86.0
    close.io = io
    args = (s["x"], s["r"], s["i"], s["A"])
    y, fs, st = m3.glr_fwd(*args, z=s["z"], init_state=s["h0"], save_states=True)
    g = m3.glr_bwd(*args, st, s["dy"], z=s["z"], dfinal=s["dfinal"], want_dinit=True)
    state = fs.clone()
    ys = m3.glr_step(state, *(s[k][:, 90] for k in ("x", "r", "i")), s["A"], z=None if s["z"] is None else s["z"][:, 90])
    assert torch.isfinite(ys).all() and torch.equal(state, fs)     # (w iota x is below a rounding)
    ref = reference(**s)
    close("y", y, ref["y"], L)
    close("final", fs, ref["final"], L)
    for k in ("dx", "dr", "di", *(("dz",) if gate else ())):
        close(k, g[k], ref[k], L)
    close("dA", g["dA"], ref["dA"], L, scale=ref["A_terms"])
    close("dinit", g["dinit"], ref["dinit"], L)


def test_decays_of_almost_nothing():
    """Decays so small that 1 - a^2 is below the smallest normal number at any gate: the
    state passes through, and no gradient is infinite."""
    s = inputs(2, 300, 6, torch.float32, True, 22)
    s["A"] = -torch.tensor([0.0, 1e-45, 1e-40, 1e-39, 5e-39, 1e-38], device=DEV)
    y, fs, st = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], init_state=s["h0"], save_states=True)
    g = m3.glr_bwd(s["x"], s["r"], s["i"], s["A"], st, s["dy"], dfinal=s["dfinal"], want_dinit=True)
    assert ((fs - s["h0"]).abs() <= 300 * 1.5e-19 * s["x"].abs().max() + U * s["h0"].abs()).all()
    assert all(torch.isfinite(v).all() for v in g.values())


def test_nonfinite_inputs_stay_in_their_channel_and_later():
    s = inputs(2, 700, 40, torch.bfloat16, False, 6)
    clean, _ = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], init_state=s["h0"])
    s["x"][1, 400, 7] = float("nan")
    s["x"][0, 130, 9] = float("inf")
    y, fs = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], init_state=s["h0"])
    spoiled = torch.zeros_like(y, dtype=torch.bool)
    spoiled[1, 400:, 7] = True
    spoiled[0, 130:, 9] = True
    assert torch.equal(y[~spoiled], clean[~spoiled]) and not torch.isfinite(y[spoiled]).any()
    assert not torch.isfinite(fs[1, 7]) and not torch.isfinite(fs[0, 9])
    assert torch.isfinite(fs).sum().item() == fs.numel() - 2


def test_same_bits_on_every_run_stream_and_shared_workspace():
    """Results do not depend on timing, on the stream, or on what the workspace
    served before."""
    big, small = inputs(3, 5000, 320, torch.bfloat16, True, 8), inputs(2, 260, 64, torch.bfloat16, False, 9)
    ws = m3.glr_workspace(big["x"], big["r"], big["i"], z=big["z"])

    def both(s, stream=None):
        y, fs, st = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], z=s["z"], init_state=s["h0"],
                               save_states=True, workspace=ws, stream=stream)
        g = m3.glr_bwd(s["x"], s["r"], s["i"], s["A"], st, s["dy"], z=s["z"], dfinal=s["dfinal"],
                       want_dinit=True, workspace=ws, stream=stream)
        return [y, fs, st, *g.values()]
    first, firsts = both(big), both(small)
    side = torch.cuda.Stream()
    for k in range(6):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got, gots = both(big), both(small)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(first + firsts, got + gots))


def test_captured_and_replayed():
    s = inputs(2, 3000, 128, torch.bfloat16, True, 12)
    ws = m3.glr_workspace(s["x"], s["r"], s["i"], z=s["z"])

    def both():
        y, fs, st = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], z=s["z"], save_states=True, workspace=ws)
        return [y, fs, *m3.glr_bwd(s["x"], s["r"], s["i"], s["A"], st, s["dy"], z=s["z"], workspace=ws).values()]
    ref = both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(4):
        for o in out:
            o.fill_(7.0)
        eager = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(ref, out, eager))


def test_wait_that_gives_up_is_counted_and_leaves_nan():
    """With a limit of one poll a tile that finds nothing gives up at once: the call
    ends, its sequence is NaN from there on, the count says so, and the next call on
    the workspace is right again."""
    s = inputs(1, 128 * 300, 64, torch.bfloat16, False, 13)
    ws = m3.glr_workspace(s["x"], s["r"], s["i"])
    args = (s["x"], s["r"], s["i"], s["A"])
    ref, _ = m3.glr_fwd(*args, workspace=ws)
    assert m3.glr_check(s["x"], s["r"], s["i"], ws) == 0
    m3.set_wait_limit(1)
    try:
        y, fs = m3.glr_fwd(*args, workspace=ws)
        n = m3.glr_check(s["x"], s["r"], s["i"], ws)
    finally:
        m3.set_wait_limit(0)
    assert n > 0 and torch.isnan(fs).any() and torch.isnan(y).any()
    again, _ = m3.glr_fwd(*args, workspace=ws)
    assert m3.glr_check(s["x"], s["r"], s["i"], ws) == 0 and torch.equal(again, ref)


@pytest.mark.parametrize("raw", [False, True])
def test_given_stream_without_a_workspace(raw):
    """`stream` as an argument, nothing else given: the workspace's clearing and the
    outputs are in that stream's order, whatever their memory held before and however
    long the current stream is at work."""
    s = inputs(2, 3000, 192, torch.bfloat16, True, 17)
    args = (s["x"], s["r"], s["i"], s["A"])

    def both(**kw):
        y, fs, st = m3.glr_fwd(*args, z=s["z"], init_state=s["h0"], save_states=True, **kw)
        return [y, fs, st, *m3.glr_bwd(*args, st, s["dy"], z=s["z"], dfinal=s["dfinal"], want_dinit=True, **kw).values()]
    ref = both()
    n = m3.glr_workspace(s["x"], s["r"], s["i"], z=s["z"]).numel()
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    work = torch.randn(4096, 4096, device=DEV)
    for _ in range(3):
        side.wait_stream(here)
        for st in (here, side):       # both streams' free memory full of other values
            with torch.cuda.stream(st):
                junk = [torch.full((m,), 171, dtype=torch.uint8, device=DEV) for m in (n, 2 * n, 16 << 20)]
                del junk
        work = work @ work * 1e-3     # (the current stream is behind)
        got = both(stream=side.cuda_stream if raw else side)
        here.wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_tickets_past_the_items_do_nothing():
    """A workspace whose ticket counter is not where a call left it: no workgroup writes
    anything, and m3_glr_check says so; cleared, it serves again."""
    s = inputs(2, 700, 48, torch.float32, False, 18)
    args, dims = (s["x"], s["r"], s["i"], s["A"]), (s["x"], s["r"], s["i"])
    ws = m3.glr_workspace(*dims)
    ref = m3.glr_fwd(*args, workspace=ws)
    for ticket in (2 * 6 * 1, 171, 0x7fffffff):      # (the call's items: 2 rows, 6 tiles, 1 group)
        ws.zero_()
        ws[:4].view(torch.int32)[0] = ticket
        before = ws.clone()
        y, fs = torch.full_like(s["x"], 7.0), torch.full((2, 48), 7.0, device=DEV)
        m3.glr_fwd(*args, out=(y, fs), workspace=ws)
        assert m3.glr_check(*dims, ws) == 12
        assert (y == 7.0).all() and (fs == 7.0).all() and torch.equal(ws[16:], before[16:])
    ws.zero_()
    got = m3.glr_fwd(*args, workspace=ws)
    assert m3.glr_check(*dims, ws) == 0 and all(torch.equal(a, b) for a, b in zip(ref, got))
