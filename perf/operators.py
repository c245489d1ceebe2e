"""The layer operators beside the Mamba-3 scan, as programs call them.

* `glr_*`: the gated linear recurrence (one decay per channel and token):
  a prompt, a training step (forward and backward), a decode step;
* `ffn_*`: the gated feed-forward block: from one token to a full batch,
  and its backward;
* `adamw_*`: the optimizer step over a model's tensors, states in fp32 or in
  8 bits.

Where `own` is false, `run` computes the operators' plain form: elementary
torch operations in fp32.  Where it is true, it calls the library.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


# --------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------

def _glr(name, kind, batch, seqlen, width, io="bf16", gate=False, packed=False, init=False):
    return dict(name=name, kind=kind, batch=batch, seqlen=seqlen, width=width, io=io, gate=gate,
                packed=packed, init=init)


def _ffn(name, kind, tokens, dmodel, dff, io="bf16", act="silu", packed=False):
    return dict(name=name, kind=kind, tokens=tokens, dmodel=dmodel, dff=dff, io=io, act=act,
                packed=packed)


def _adamw(name, layers, dmodel, dff, states="f32", grad="f32", low=False, pad=True, step=1000):
    return dict(name=name, kind="adamw", layers=layers, dmodel=dmodel, dff=dff, states=states,
                grad=grad, low=low, pad=pad, step=step)


def listed():
    return [
        # a serving batch's token through the recurrence, gated: launch latency
        _glr("glr_decode", "glr_step", 64, 1, 4096, gate=True),
        # prompts of a serving batch, inputs as slices of one projection's output
        _glr("glr_prefill", "glr_fwd", 4, 2048, 4096, gate=True, packed=True, init=True),
        # one long document in training
        _glr("glr_train_long", "glr_train", 1, 65536, 2048),
        # a small fp32 run of odd sizes with the gate, started from a state
        _glr("glr_train_fp32", "glr_train", 3, 1001, 1000, io="f32", gate=True, init=True),
        # one token of one sequence: the weights are streamed once
        _ffn("ffn_decode_one", "ffn_fwd", 1, 2048, 8192),
        # a serving batch's tokens
        _ffn("ffn_decode_batch", "ffn_fwd", 48, 2048, 8192, act="gelu"),
        # a batch of prompts
        _ffn("ffn_prefill", "ffn_fwd", 8192, 2048, 8192, packed=True),
        # a training step's backward
        _ffn("ffn_backward", "ffn_bwd", 8192, 2048, 8192),
        # a small fp32 run of odd sizes, backward
        _ffn("ffn_backward_fp32", "ffn_bwd", 777, 1000, 2730, io="f32", act="gelu"),
        # a small model's many small tensors, back to back in one buffer
        _adamw("adamw_small", 12, 129, 344, pad=False, step=3),
        # four layers of a wide stack
        _adamw("adamw_fp32", 4, 2048, 8192),
        # the same with 8-bit states, bf16 gradients and a bf16 copy of the weights
        _adamw("adamw_8bit", 4, 2048, 8192, states="8bit", grad="bf16", low=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: mostly a multiple of 64 or 8, sometimes any number."""
    unit = rng.choice([64, 64, 8, 8, 2, 1])
    n = max(1, _log_int(rng, lo, hi) // unit) * unit
    return n + unit if n == 3 << 10 else n


def draw(rng):
    kind = rng.choice(["glr_fwd", "glr_train", "glr_step", "ffn_fwd", "ffn_fwd", "ffn_bwd", "adamw"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind.startswith("glr"):
        width = _width(rng, 64, 8192)
        most = (1 << 27 if kind == "glr_train" else 1 << 26) // width // (2 if io == "f32" else 1)
        gate, init = rng.random() < 0.5, rng.random() < 0.5
        if kind == "glr_step":
            c = _glr("", kind, _log_int(rng, 1, 512), 1, width, io, gate)
        else:
            if kind == "glr_train" and gate:
                most //= 2
            tokens = _log_int(rng, 64, most)
            seqlen = _log_int(rng, max(1, tokens // 64), min(tokens, 65536))
            c = _glr("", kind, max(1, tokens // seqlen), seqlen, width, io, gate,
                     rng.random() < 0.5, init)
    elif kind.startswith("ffn"):
        dmodel, dff = _width(rng, 256, 4096), 0
        dff = _width(rng, max(256, dmodel), 4 * dmodel)
        dff = min(dff, 11008)
        most = min(16384, (1 << 37) // (dmodel * dff)) // (16 if io == "f32" else 1)
        c = _ffn("", kind, _log_int(rng, 1 if kind == "ffn_fwd" else 64, max(64, most)), dmodel, dff,
                 io, rng.choice(["silu", "gelu"]), kind == "ffn_fwd" and rng.random() < 0.5)
    else:
        dmodel = _width(rng, 64, 2048)
        dff = min(_width(rng, dmodel, 4 * dmodel), 8192)
        layers = _log_int(rng, 1, 24)
        layers = max(1, min(layers, (250 << 20) // (3 * dmodel * dff + 4 * dmodel * dmodel)))
        c = _adamw("", layers, dmodel, dff, rng.choice(["f32", "8bit"]),
                   rng.choice(["f32", "bf16"]), rng.random() < 0.5, rng.random() < 0.5,
                   _log_int(rng, 1, 100000))
    del c["name"]
    return c


def _shapes(c):
    """The tensors of a stack of mixers and feed-forward blocks: matrices and vectors."""
    d, f = c["dmodel"], c["dff"]
    return [(d, d)] * 4 * c["layers"] + [(f, d)] * 2 * c["layers"] + [(d, f)] * c["layers"] \
        + [(d,)] * 4 * c["layers"]


def work(c):
    e = 4 if c.get("io") == "f32" else 2
    if c["kind"] == "glr_step":
        n = c["batch"] * c["width"]
        return {"bytes": n * ((4 + c["gate"]) * e + 8) + 4 * c["width"], "flops": 40 * n}
    if c["kind"] in ("glr_fwd", "glr_train"):
        n, s = c["batch"] * c["seqlen"] * c["width"], 4 * c["batch"] * c["width"]
        b = n * (4 + c["gate"]) * e + s * (1 + c["init"]) + 4 * c["width"]
        if c["kind"] == "glr_train":
            b += n * (7 + 2 * c["gate"]) * e + s * (2 + c["init"]) + 8 * c["width"]
        return {"bytes": b, "flops": (40 if c["kind"] == "glr_fwd" else 120) * n}
    if c["kind"] in ("ffn_fwd", "ffn_bwd"):
        t, d, f = c["tokens"], c["dmodel"], c["dff"]
        if c["kind"] == "ffn_fwd":
            return {"bytes": e * (2 * t * d + 3 * d * f), "flops": 6 * t * d * f}
        # dh, dx (two), three weight gradients, and g and u formed again
        return {"bytes": e * (3 * t * d + 6 * d * f), "flops": 16 * t * d * f}
    n = sum(math.prod(s) for s in _shapes(c))
    b = 8 + (4 if c["grad"] == "f32" else 2) + (2 if c["low"] else 0)
    b += 16 if c["states"] == "f32" else 4 + 16 / 256
    return {"bytes": n * b, "flops": 14 * n}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(DEV).manual_seed(int(seed))


def _randn(gen, *shape, io=torch.float32, scale=1.0):
    return (torch.randn(shape, device=DEV, generator=gen) * scale).to(io)


def _prepare_glr(c, gen):
    io, step = IO[c["io"]], c["kind"] == "glr_step"
    B, L, D = c["batch"], c["seqlen"], c["width"]
    n = 4 if c["gate"] else 3
    lead = (B,) if step else (B, L)
    if c["packed"]:
        parts = _randn(gen, *lead, n * D, io=io).split(D, dim=-1)
    else:
        parts = [_randn(gen, *lead, D, io=io) for _ in range(n)]
    # log-decays at an open gate: memories of one to a hundred and fifty tokens
    u = torch.rand((D,), device=DEV, generator=gen)
    s = dict(x=parts[0], r=parts[1], i=parts[2], z=parts[3] if c["gate"] else None,
             A=-torch.exp(math.log(0.0066) + u * math.log(1.0 / 0.0066)))
    s["h0"] = _randn(gen, B, D) if c["init"] or step else None
    if c["kind"] == "glr_train":
        s["dy"] = _randn(gen, B, L, D, io=io)
        s["dfinal"] = _randn(gen, B, D)
    return s


def _prepare_ffn(c, gen):
    io = IO[c["io"]]
    T, D, F = c["tokens"], c["dmodel"], c["dff"]
    x = _randn(gen, T, 2 * D if c["packed"] else D, io=io)
    s = dict(x=x[:, :D], act=c["act"],
             Wg=_randn(gen, F, D, io=io, scale=D ** -0.5), Wu=_randn(gen, F, D, io=io, scale=D ** -0.5),
             Wd=_randn(gen, D, F, io=io, scale=F ** -0.5))
    if c["kind"] == "ffn_bwd":
        s["dy"] = _randn(gen, T, D, io=io)
    return s


BLOCK = 256          # elements that share a scale of the 8-bit states


def _prepare_adamw(c, gen):
    shapes = _shapes(c)
    unit = 16 if c["pad"] else 1
    sizes = [math.prod(s) for s in shapes]
    room = [-(-n // unit) * unit for n in sizes]
    total = sum(room)
    at = [0]
    for n in room:
        at.append(at[-1] + n)

    def flat(io=torch.float32, scale=1.0):
        return _randn(gen, total, io=io, scale=scale)

    def views(t):
        return [t[at[k]:at[k] + n].view(shapes[k]) for k, n in enumerate(sizes)]

    p, g = flat(scale=0.02), flat(IO[c["grad"]], 1e-3)
    s = dict(step=c["step"], lr=3e-4, betas=(0.9, 0.95), eps=1e-8,
             wd=[0.1 if len(x) > 1 else 0.0 for x in shapes],
             # the coefficient that clips the gradients' norm, as its reduction left it
             grad_scale=torch.full((1,), 0.37, device=DEV), seed=12345 + c["step"],
             flat=dict(p=p), p=views(p), g=views(g))
    if c["low"]:
        s["flat"]["low"] = torch.zeros(total, dtype=torch.bfloat16, device=DEV)
        s["low"] = views(s["flat"]["low"])
    m, v = flat(scale=3e-4), flat(scale=4e-4).square_()
    if c["states"] == "f32":
        s["flat"].update(m=m, v=v)
        s.update(m=views(m), v=views(v))
    else:
        blocks = [-(-n // BLOCK) for n in sizes]
        m8 = torch.zeros(total, dtype=torch.float8_e4m3fn, device=DEV)
        v8 = torch.zeros(total, dtype=torch.float8_e4m3fn, device=DEV)
        scales = torch.zeros((sum(blocks), 2), device=DEV)
        s["flat"].update(m=m8, v=v8, scales=scales)
        s.update(m=views(m8), v=views(v8), scales=list(scales.split(blocks)))
        for k, (mk, vk) in enumerate(zip(views(m), views(v))):
            for col, (to, w) in enumerate(((s["m"][k], mk), (s["v"][k], vk.sqrt()))):
                w, n = _blocks(w)
                sc = w.abs().amax(1, keepdim=True) / 448.0
                s["scales"][k][:, col:col + 1] = sc
                to.view(-1).copy_((w / sc).reshape(-1)[:n].to(torch.float8_e4m3fn))
    return s


def prepare(c, seed):
    gen = _gen(seed)
    make = _prepare_glr if c["kind"].startswith("glr") else _prepare_ffn if c["kind"].startswith("ffn") \
        else _prepare_adamw
    s = make(c, gen)
    s["kind"] = c["kind"]
    return s


# --------------------------------------------------------------------------
# Plain forms
# --------------------------------------------------------------------------

def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along axis 1, the affine maps of 1, 2, 4, ... tokens joined."""
    d = 1
    while d < a.shape[1]:   # log2(L) passes over the whole arrays
        b = torch.cat((b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]), 1)
        a = torch.cat((a[:, :d], a[:, d:] * a[:, :-d]), 1)
        d *= 2
    return b


def _gates(s):
    x, r, i = s["x"].float(), s["r"].float(), s["i"].float()
    rho, iota = _sigmoid(r), _sigmoid(i)
    la = s["A"] * rho
    return x, rho, iota, torch.exp(la), torch.sqrt(-torch.expm1(2.0 * la))


def _plain_step(s):
    x, rho, iota, a, w = _gates(s)
    h = a * s["h0"] + w * iota * x
    s["h0"].copy_(h)
    if s["z"] is not None:
        z = s["z"].float()
        h = h * (z * _sigmoid(z))
    return dict(y=h.to(s["x"].dtype), state=s["h0"])


def _plain_glr(s):
    x, rho, iota, a, w = _gates(s)
    b = w * iota * x
    if s["h0"] is not None:
        b[:, 0] += a[:, 0] * s["h0"]
    h = _scan(a, b)
    io = s["x"].dtype
    gate = 1.0
    if s["z"] is not None:
        z = s["z"].float()
        sz = _sigmoid(z)
        gate = z * sz
    out = dict(y=(h * gate).to(io), final=h[:, -1].clone())
    if s["kind"] == "glr_fwd":
        return out
    dy = s["dy"].float()
    dh = dy * gate
    dh[:, -1] += s["dfinal"]
    # g_t = dh_t + a_{t+1} g_{t+1}: the same scan from the last token to the first
    g = _scan(torch.cat((torch.ones_like(a[:, :1]), a[:, 1:].flip(1)), 1), dh.flip(1)).flip(1)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros_like(h[:, 0])
    prev = torch.cat((h0[:, None], h[:, :-1]), 1)
    dla = a * g * prev - (a * a / w) * (g * iota * x)
    out.update(dx=(g * w * iota).to(io), di=(g * w * x * iota * (1.0 - iota)).to(io),
               dr=(s["A"] * dla * rho * (1.0 - rho)).to(io), dA=(rho * dla).sum((0, 1)))
    if s["h0"] is not None:
        out["dinit"] = a[:, 0] * g[:, 0]
    if s["z"] is not None:
        out["dz"] = (dy * h * (sz + gate * (1.0 - sz))).to(io)
    return out


def _act(g, act):
    """act(g) = g sigmoid(p) and its derivative; p = g (SiLU) or the cubic of the tanh form of GELU."""
    if act == "silu":
        s = _sigmoid(g)
        return g * s, s + g * s * (1.0 - s)
    k = 2.0 * math.sqrt(2.0 / math.pi)
    s = _sigmoid(k * (g + 0.044715 * g * g * g))
    return g * s, s + g * s * (1.0 - s) * (k + 3.0 * 0.044715 * k * g * g)


def _plain_ffn(s):
    x, wg, wu, wd = (s[k].float() for k in ("x", "Wg", "Wu", "Wd"))
    io = s["x"].dtype
    g, u = x @ wg.T, x @ wu.T
    f, df = _act(g, s["act"])
    if s["kind"] == "ffn_fwd":
        return dict(y=((f * u) @ wd.T).to(io))
    dy = s["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * df, dh * f
    return dict(dx=(dg @ wg + du @ wu).to(io), dWg=(dg.T @ x).to(io), dWu=(du.T @ x).to(io),
                dWd=(dy.T @ (f * u)).to(io))


def _blocks(t):
    """A tensor's elements in rows of BLOCK, zeros past its end, and their count."""
    n = t.numel()
    return torch.nn.functional.pad(t.reshape(-1), (0, -n % BLOCK)).view(-1, BLOCK), n


def _noise(n, seed):
    """Two 16-bit uniform numbers for each element, from its index and the step's seed."""
    i = torch.arange(n, device=DEV) & 0xffffffff
    h = ((i ^ (seed & 0xffffffff)) * 0x9E3779B1) & 0xffffffff
    h = ((h ^ (h >> 15)) * 0x6A09E667) & 0xffffffff
    h = ((h ^ (h >> 13)) * 0x9E3779B1) & 0xffffffff
    h = h ^ (h >> 16)
    return h & 0xffff, h >> 16


def _round8(w, u):
    """|w| <= 448 to e4m3, up with a probability of the part cut off: u is 16 uniform bits."""
    a = w.abs()
    big = ((a.view(torch.int32) + (u << 4).to(torch.int32)) & ~0xfffff).view(torch.float32)
    small = torch.floor(a * 512.0 + u.float() * 2.0 ** -16) * 2.0 ** -9
    q = torch.where(a >= 2.0 ** -6, big, small).clamp(max=448.0)
    return torch.where(w < 0, -q, q)


def _adamw_one(s, k):
    p, g = s["p"][k], s["g"][k].float() * s["grad_scale"]
    b1, b2 = s["betas"]
    f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    bc1, bc2 = 1.0 - b1 ** s["step"], 1.0 - b2 ** s["step"]
    eight = "scales" in s
    if eight:
        sc = s["scales"][k]
        (m, n), (rv, _) = _blocks(s["m"][k].float()), _blocks(s["v"][k].float())
        m = (m * sc[:, :1]).view(-1)[:n].view(p.shape)
        rv = (rv * sc[:, 1:]).view(-1)[:n].view(p.shape)
        v = rv * rv
    else:
        m, v = s["m"][k], s["v"][k]
    m = m * f32(b1) + g * f32(1.0 - b1)
    v = v * f32(b2) + (g * g) * f32(1.0 - b2)
    root = torch.sqrt(v)
    p.copy_(p * f32(1.0 - s["lr"] * s["wd"][k])
            - (m * f32(s["lr"] / bc1)) / (root * f32(bc2 ** -0.5) + f32(s["eps"])))
    if "low" in s:
        s["low"][k].copy_(p)
    if not eight:
        s["m"][k].copy_(m)
        s["v"][k].copy_(v)
        return
    um, uv = _noise(n, s["seed"] + k)
    for col, (to, w, u) in enumerate(((s["m"][k], m, um), (s["v"][k], root, uv))):
        w, _ = _blocks(w)
        most = w.abs().amax(1, keepdim=True)
        scale = most * f32(1.0 / 448.0)
        sc[:, col:col + 1] = scale
        q = _round8((w * torch.where(most > 0, 1.0 / scale, 0.0)).reshape(-1)[:n], u)
        if col == 1:   # a second moment that is not zero is not stored as zero
            q = torch.where(root.reshape(-1) > 0, q.clamp(min=2.0 ** -9), q)
        to.view(-1).copy_(q.to(torch.float8_e4m3fn))


def _plain_adamw(s):
    [_adamw_one(s, k) for k in range(len(s["p"]))]
    return s["flat"]


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def _own(s):
    from paper_2603_15569_amd import m3

    kind = s["kind"]
    if kind == "glr_step":
        return dict(y=m3.glr_step(s["h0"], s["x"], s["r"], s["i"], s["A"], z=s["z"]), state=s["h0"])
    if kind in ("glr_fwd", "glr_train"):
        if "ws" not in s:   # a program keeps its workspace
            s["ws"] = m3.glr_workspace(s["x"], s["r"], s["i"], z=s["z"])
        fwd = m3.glr_fwd(s["x"], s["r"], s["i"], s["A"], z=s["z"], init_state=s["h0"],
                         save_states=kind == "glr_train", workspace=s["ws"])
        out = dict(y=fwd[0], final=fwd[1])
        if kind == "glr_train":
            out.update(m3.glr_bwd(s["x"], s["r"], s["i"], s["A"], fwd[2], s["dy"], z=s["z"],
                                  dfinal=s["dfinal"], want_dinit=s["h0"] is not None,
                                  workspace=s["ws"]))
        return out
    if kind in ("ffn_fwd", "ffn_bwd"):
        if "ws" not in s:
            s["ws"] = m3.ffn_workspace(s["x"], s["Wg"], backward=kind == "ffn_bwd")
        if kind == "ffn_fwd":
            return dict(y=m3.ffn_fwd(s["x"], s["Wg"], s["Wu"], s["Wd"], act=s["act"],
                                     workspace=s["ws"]))
        return m3.ffn_bwd(s["x"], s["Wg"], s["Wu"], s["Wd"], s["dy"], act=s["act"],
                          workspace=s["ws"])
    if "table" not in s:   # a program builds its table once and keeps it
        s["table"] = m3.adamw_table(s["p"], s["g"], s["m"], s["v"], weight_decay=s["wd"],
                                    low=s.get("low"), scales=s.get("scales"))
    m3.adamw_step(s["table"], step=s["step"], lr=s["lr"], betas=s["betas"], eps=s["eps"],
                  grad_scale=s["grad_scale"], seed=s["seed"])
    return s["flat"]


def run(s):
    if own:
        return _own(s)
    if s["kind"] == "glr_step":
        return _plain_step(s)
    if s["kind"].startswith("glr"):
        return _plain_glr(s)
    if s["kind"].startswith("ffn"):
        return _plain_ffn(s)
    return _plain_adamw(s)


# --------------------------------------------------------------------------
# The definitions in 64 bits
# --------------------------------------------------------------------------

def _exact_glr(c, s):
    leaf = {k: s[k].double().requires_grad_() for k in ("x", "r", "i", "A")}
    rho = torch.sigmoid(leaf["r"])
    la = leaf["A"] * rho
    a = la.exp()
    b = torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(leaf["i"]) * leaf["x"]
    step = c["kind"] == "glr_step"
    if step:
        a, b = a[:, None], b[:, None]
    B, L, D = a.shape
    ad, bd = a.detach(), b.detach()
    # token by token, from the definition
    h = torch.empty((B, L, D), dtype=torch.float64, device=DEV)
    cur = torch.zeros((B, D), dtype=torch.float64, device=DEV) if s["h0"] is None else s["h0"].double()
    first = cur
    for t in range(L):
        cur = torch.addcmul(bd[:, t], ad[:, t], cur, out=h[:, t])
    silu = torch.ones((), dtype=torch.float64, device=DEV)
    if s["z"] is not None:
        z = s["z"].double().requires_grad_()
        silu = torch.nn.functional.silu(z)
        silu = silu[:, None] if step else silu
    y = h * silu.detach()
    if step:
        return dict(y=y[:, 0], state=h[:, 0])
    out = dict(y=y, final=h[:, -1])
    if c["kind"] == "glr_fwd":
        return out
    dy = s["dy"].double()
    dh = dy * silu.detach()
    dh[:, -1] += s["dfinal"].double()
    for t in range(L - 2, -1, -1):
        dh[:, t].addcmul_(ad[:, t + 1], dh[:, t + 1])
    prev = torch.cat((first[:, None], h[:, :-1]), 1)
    torch.autograd.backward([a, b], [dh * prev, dh])
    out.update(dx=leaf["x"].grad, dr=leaf["r"].grad, di=leaf["i"].grad, dA=leaf["A"].grad)
    if s["h0"] is not None:
        out["dinit"] = ad[:, 0] * dh[:, 0]
    if s["z"] is not None:
        silu.backward(dy * h)
        out["dz"] = z.grad
    return out


def _exact_ffn(c, s):
    x, wg, wu, wd = (s[k].double().requires_grad_(c["kind"] == "ffn_bwd") for k in ("x", "Wg", "Wu", "Wd"))
    f = torch.nn.functional
    g, u = f.linear(x, wg), f.linear(x, wu)
    y = f.linear((f.silu(g) if c["act"] == "silu" else f.gelu(g, approximate="tanh")) * u, wd)
    if c["kind"] == "ffn_fwd":
        return dict(y=y)
    y.backward(s["dy"].double())
    return dict(dx=x.grad, dWg=wg.grad, dWu=wu.grad, dWd=wd.grad)


def _exact_adamw(c, s):
    b1, b2 = s["betas"]
    ext = {k: v.double().clone() for k, v in s["flat"].items()}
    row = 0
    for k, p in enumerate(s["p"]):
        n = p.numel()
        at = p.storage_offset()
        m, v, g = s["m"][k].double().view(-1), s["v"][k].double().view(-1), s["g"][k].double().view(-1)
        g = g * s["grad_scale"].double()
        if "scales" in s:
            by = s["scales"][k].double().repeat_interleave(BLOCK, 0)[:n]
            m, v = m * by[:, 0], (v * by[:, 1]) ** 2
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        mh, vh = m / (1 - b1 ** s["step"]), v / (1 - b2 ** s["step"])
        new = p.double().view(-1) * (1 - s["lr"] * s["wd"][k]) - s["lr"] * mh / (vh.sqrt() + s["eps"])
        ext["p"][at:at + n] = new
        if "low" in ext:
            ext["low"][at:at + n] = new
        if "scales" in s:
            for col, w in enumerate((m.abs(), v.sqrt())):
                w = torch.nn.functional.pad(w, (0, -n % BLOCK)).view(-1, BLOCK)
                ext["scales"][row:row + len(w), col] = w.amax(1) / 448
            row += len(w)
        else:
            ext["m"][at:at + n], ext["v"][at:at + n] = m, v
    if "scales" in s:   # the rounding's numbers decide the codes: they have no value in 64 bits
        ext["m"] = ext["v"] = None
    return ext


def exact(c, seed):
    s = prepare(c, seed)
    how = _exact_glr if c["kind"].startswith("glr") else _exact_ffn if c["kind"].startswith("ffn") else _exact_adamw
    return how(c, s)
