"""CPU tests of the operators beside the scan: the refusals of the C ABI (every
argument error is caught on the host before a launch) and of the binding, the
workspace queries, and the optimizer's table."""
import ctypes

import pytest
import torch

from paper_2603_15569_amd import m3

FAKE = 0x100000   # 16-byte aligned fake device address; never dereferenced


@pytest.fixture(scope="module")
def L():
    return m3.lib()


def glr(**kw):
    d = dict(batch=2, seqlen=300, width=64, io=m3.M3_BF16, flags=0)
    for t in "xriz":
        d[t + "_stride_b"], d[t + "_stride_t"] = 300 * 64, 64
    d.update(kw)
    return m3.M3GlrDims(**d)


def fwd(L, d, over=None, wsb=None):
    p = [FAKE] * 9               # x r i A z init y final states
    p[4] = p[5] = p[8] = None
    for k, v in (over or {}).items():
        p[k] = v
    need = L.m3_glr_workspace_bytes(ctypes.byref(d)) if d is not None else 0
    ws = FAKE if not over or "ws" not in over else over["ws"]
    return L.m3_glr_fwd(ctypes.byref(d) if d is not None else None, *p[:9], ws, need if wsb is None else wsb, None)


def test_glr_refusals(L):
    assert fwd(L, None) == m3.M3_ERR_NULL
    assert fwd(L, glr(io=5)) == m3.M3_ERR_DTYPE
    for bad in (dict(batch=0), dict(width=0), dict(seqlen=-1), dict(flags=1), dict(x_stride_t=-1),
                dict(r_stride_t=1 << 24), dict(width=1 << 24), dict(batch=1 << 20, seqlen=1 << 20, width=1 << 20),
                dict(i_stride_b=1 << 62)):
        assert fwd(L, glr(**bad)) == m3.M3_ERR_SHAPE, bad
        assert L.m3_glr_workspace_bytes(ctypes.byref(glr(**bad))) == 0, bad
    for k in (0, 1, 2, 3, 6, 7):
        assert fwd(L, glr(), {k: None}) == m3.M3_ERR_NULL, k
    assert fwd(L, glr(), {0: FAKE + 1}) == m3.M3_ERR_ALIGN
    assert fwd(L, glr(), {4: FAKE + 1}) == m3.M3_ERR_ALIGN
    assert fwd(L, glr(), {3: FAKE + 2}) == m3.M3_ERR_ALIGN
    assert fwd(L, glr(), {8: FAKE + 2}) == m3.M3_ERR_ALIGN
    assert fwd(L, glr(io=m3.M3_F32), {0: FAKE + 2}) == m3.M3_ERR_ALIGN
    assert fwd(L, glr(), wsb=16) == m3.M3_ERR_WORKSPACE
    need = L.m3_glr_workspace_bytes(ctypes.byref(glr()))
    assert need >= 256 + 4 * 2 * 3 * 64 * 8 and fwd(L, glr(), wsb=need - 1) == m3.M3_ERR_WORKSPACE

    def bwd(d, over=None):
        p = [FAKE] * 14          # x r i A z states dy dfinal dx dr di dz dA dinit
        for k in (4, 7, 11, 13):
            p[k] = None
        for k, v in (over or {}).items():
            p[k] = v
        return L.m3_glr_bwd(ctypes.byref(d), *p, FAKE, need, None)
    for k in (0, 1, 2, 3, 5, 6, 8, 9, 10, 12):
        assert bwd(glr(), {k: None}) == m3.M3_ERR_NULL, k
    assert bwd(glr(), {4: FAKE}) == m3.M3_ERR_NULL          # the gate without room for its gradient
    assert bwd(glr(), {9: FAKE + 1}) == m3.M3_ERR_ALIGN
    assert bwd(glr(), {12: FAKE + 2}) == m3.M3_ERR_ALIGN

    def step(d, over=None):
        p = [FAKE] * 7           # state x r i A z y
        p[5] = None
        for k, v in (over or {}).items():
            p[k] = v
        return L.m3_glr_step(ctypes.byref(d), *p, None)
    for k in (0, 1, 2, 3, 4, 6):
        assert step(glr(), {k: None}) == m3.M3_ERR_NULL, k
    assert step(glr(), {0: FAKE + 2}) == m3.M3_ERR_ALIGN
    assert step(glr(batch=1 << 20, width=1 << 20)) == m3.M3_ERR_SHAPE
    n = ctypes.c_uint32(9)
    assert L.m3_glr_check(ctypes.byref(glr()), FAKE, need, None, None) == m3.M3_ERR_NULL
    assert L.m3_glr_check(ctypes.byref(glr()), FAKE, 16, ctypes.byref(n), None) == m3.M3_ERR_WORKSPACE
    assert n.value == 9
    assert L.m3_glr_check(ctypes.byref(glr(seqlen=m3.GLR_CHUNK)), FAKE, need, ctypes.byref(n), None) == m3.M3_OK
    assert n.value == 0          # (one run of tokens: nothing waits)
    assert L.m3_last_hip_error() == 0


def ffn(**kw):
    d = dict(tokens=100, dmodel=64, dff=160, io=m3.M3_BF16, act=0, x_stride=64, dy_stride=64)
    d.update(kw)
    return m3.M3FfnDims(**d)


def test_ffn_refusals(L):
    def call(d, over=None, wsb=None, ws=FAKE):
        p = [FAKE] * 5           # x Wg Wu Wd y
        for k, v in (over or {}).items():
            p[k] = v
        need = L.m3_ffn_workspace_bytes(ctypes.byref(d), 0) if d is not None else 0
        return L.m3_ffn_fwd(ctypes.byref(d) if d is not None else None, *p, ws, need if wsb is None else wsb, None)
    assert call(None) == m3.M3_ERR_NULL
    assert call(ffn(io=9)) == m3.M3_ERR_DTYPE
    for bad in (dict(tokens=-1), dict(dmodel=0), dict(dff=0), dict(act=2), dict(x_stride=63), dict(dmodel=1 << 17, x_stride=1 << 17),
                dict(dff=1 << 17), dict(x_stride=1 << 21), dict(tokens=1 << 40)):
        assert call(ffn(**bad)) == m3.M3_ERR_SHAPE, bad
        assert L.m3_ffn_workspace_bytes(ctypes.byref(ffn(**bad)), 1) == 0, bad
    assert L.m3_ffn_workspace_bytes(ctypes.byref(ffn(dy_stride=3)), 0) > 0
    assert L.m3_ffn_workspace_bytes(ctypes.byref(ffn(dy_stride=3)), 1) == 0
    for k in range(5):
        assert call(ffn(), {k: None}) == m3.M3_ERR_NULL, k
    assert call(ffn(), {1: FAKE + 2}) == m3.M3_ERR_ALIGN         # whole pieces: 16 bytes
    assert call(ffn(), {3: FAKE + 8}) == m3.M3_ERR_ALIGN
    assert call(ffn(dmodel=65, x_stride=65), {1: FAKE + 1}) == m3.M3_ERR_ALIGN
    assert call(ffn(), {0: FAKE + 1}) == m3.M3_ERR_ALIGN
    assert call(ffn(), ws=FAKE + 4) == m3.M3_ERR_ALIGN
    assert call(ffn(), ws=None) == m3.M3_ERR_WORKSPACE
    assert call(ffn(), wsb=1024) == m3.M3_ERR_WORKSPACE
    assert call(ffn(tokens=0), {0: None, 4: None}) == m3.M3_OK   # nothing to do, nothing launched

    def bwd(d, over=None):
        p = [FAKE] * 9           # x Wg Wu Wd dy dx dWg dWu dWd
        for k, v in (over or {}).items():
            p[k] = v
        return L.m3_ffn_bwd(ctypes.byref(d), *p, FAKE, L.m3_ffn_workspace_bytes(ctypes.byref(d), 1), None)
    for k in range(9):
        assert bwd(ffn(), {k: None}) == m3.M3_ERR_NULL, k
    assert bwd(ffn(), {6: FAKE + 1}) == m3.M3_ERR_ALIGN
    assert L.m3_last_hip_error() == 0


def plan(L, tensors, gtype=m3.M3_F32, flags=0, table=None, nbytes=0):
    arr = (m3.M3AdamwTensor * max(len(tensors), 1))(*tensors)
    p = m3.M3AdamwPlan()
    return L.m3_adamw_plan_make(arr, len(tensors), gtype, flags, ctypes.byref(p), table, nbytes), p


def tensor(n=1000, decay=0.1, **kw):
    d = dict(p=FAKE, g=FAKE, m=FAKE, v=FAKE, low=None, scales=None)
    d.update(kw)
    return m3.M3AdamwTensor(*[d[k] for k in ("p", "g", "m", "v", "low", "scales")], n, decay)


def test_adamw_refusals(L):
    for k in ("p", "g", "m", "v"):
        assert plan(L, [tensor(**{k: None})])[0] == m3.M3_ERR_NULL, k
    assert plan(L, [tensor()], flags=m3.M3_ADAMW_8BIT)[0] == m3.M3_ERR_NULL      # no scales
    assert plan(L, [tensor(n=0, p=None)])[0] == m3.M3_OK
    assert plan(L, [tensor()], gtype=3)[0] == m3.M3_ERR_DTYPE
    assert plan(L, [tensor()], flags=2)[0] == m3.M3_ERR_SHAPE
    assert plan(L, [tensor(n=-1)])[0] == m3.M3_ERR_SHAPE
    assert plan(L, [tensor(decay=float("nan"))])[0] == m3.M3_ERR_SHAPE
    assert plan(L, [tensor(n=1 << 40)])[0] == m3.M3_ERR_SHAPE
    for k in ("p", "g", "m", "v"):
        assert plan(L, [tensor(**{k: FAKE + 2})])[0] == m3.M3_ERR_ALIGN, k
    assert plan(L, [tensor(g=FAKE + 2)], gtype=m3.M3_BF16)[0] == m3.M3_OK
    assert plan(L, [tensor(m=FAKE + 1, v=FAKE + 3, scales=FAKE)], flags=m3.M3_ADAMW_8BIT)[0] == m3.M3_OK
    assert plan(L, [tensor(low=FAKE + 1)])[0] == m3.M3_ERR_ALIGN
    _, p = plan(L, [tensor()])

    def step(table=FAKE, pl=p, gs=None, **kw):
        c = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, seed=0)
        c.update(kw)
        c = m3.M3AdamwConfig(*[c[k] for k in ("lr", "beta1", "beta2", "eps", "step", "seed")])
        return L.m3_adamw_step(ctypes.byref(c), ctypes.byref(pl) if pl is not None else None, table, gs, None)
    assert step(pl=None) == m3.M3_ERR_NULL and step(table=None) == m3.M3_ERR_NULL
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1.0),
                dict(eps=float("inf")), dict(lr=float("nan"))):
        assert step(**bad) == m3.M3_ERR_SHAPE, bad
    assert step(gs=FAKE + 2) == m3.M3_ERR_ALIGN and step(table=FAKE + 8) == m3.M3_ERR_ALIGN
    _, none = plan(L, [tensor(n=0, p=None)])
    assert (none.rows, none.groups) == (0, 0) and step(pl=none, table=None) == m3.M3_OK
    assert L.m3_last_hip_error() == 0


def test_adamw_table(L):
    """Workgroups of 1024 elements; the table's rows skip empty tensors and its map
    names each workgroup's row; a buffer below the plan's size is refused."""
    ts = [tensor(n=1), tensor(n=0), tensor(n=1024), tensor(n=1025, decay=0.0), tensor(n=5000)]
    s, p = plan(L, ts)
    assert s == m3.M3_OK and (p.rows, p.groups) == (4, 1 + 1 + 2 + 5) and p.bytes >= 4 * 72 + 9 * 4
    buf = torch.zeros(p.bytes + 8, dtype=torch.uint8)
    buf[p.bytes:] = 7
    assert plan(L, ts, table=buf.data_ptr(), nbytes=p.bytes - 1)[0] == m3.M3_ERR_WORKSPACE
    assert plan(L, ts, table=buf.data_ptr(), nbytes=p.bytes)[0] == m3.M3_OK
    assert (buf[p.bytes:] == 7).all()
    words = buf[:p.bytes].view(torch.int32)
    row = 72 // 4
    assert words[4 * row:4 * row + 9].tolist() == [0, 1, 2, 2, 3, 3, 3, 3, 3]
    assert [words[k * row + 12:k * row + 16].tolist() for k in range(4)] == \
        [[0, 1, 1, 0], [1, 1, 1024, 2], [2, 2, 1, 3], [4, 5, 904, 4]]


def test_binding_refusals():
    """The binding's own checks, before any call of the library."""
    x = torch.zeros(2, 5, 8, dtype=torch.bfloat16)
    A = -torch.ones(8)
    ok = m3.glr_dims(x, x, x, x)
    assert (ok.batch, ok.seqlen, ok.width, ok.x_stride_b, ok.x_stride_t) == (2, 5, 8, 40, 8)
    one = m3.glr_dims(x[:1, :, :], x[1:], x[:1])
    assert one.x_stride_b == 0 and one.r_stride_t == 8     # (a stride over one row is never walked)
    packed = torch.zeros(2, 5, 24, dtype=torch.bfloat16).split(8, -1)
    assert m3.glr_dims(*packed).i_stride_t == 24
    for bad in (x.float(), x[:, :4], x[:, :, :4]):
        with pytest.raises(ValueError):
            m3.glr_fwd(x, bad, x, A, workspace=x)
    with pytest.raises(ValueError):
        m3.glr_dims(x.half())
    with pytest.raises(ValueError):
        m3.glr_dims(x.transpose(1, 2))
    with pytest.raises(ValueError):
        m3.glr_fwd(x, x, x, A.double(), workspace=x)
    with pytest.raises(ValueError):
        m3.glr_fwd(x, x, x, A[:4], workspace=x)
    with pytest.raises(ValueError):
        m3.glr_bwd(x, x, x, A, torch.zeros(2, 1, 8), x[:1], workspace=x)
    with pytest.raises(ValueError):
        m3.glr_bwd(x, x, x, A, torch.zeros(2, 2, 8), x, workspace=x)
    with pytest.raises(ValueError):
        m3.glr_step(torch.zeros(2, 8), x, x, x, A)
    W, Wd = torch.zeros(12, 8, dtype=torch.bfloat16), torch.zeros(8, 12, dtype=torch.bfloat16)
    for args in ((x, W, W, W), (x, W.float(), W, Wd), (x, W, W[:3], Wd), (x.half(), W, W, Wd),
                 (x.transpose(0, 1), W, W, Wd)):
        with pytest.raises(ValueError):
            m3.ffn_fwd(*args, workspace=x)
    with pytest.raises(ValueError):
        m3.ffn_fwd(x, W, W, Wd, act="relu", workspace=x)
    with pytest.raises(ValueError):
        m3.ffn_bwd(x, W, W, Wd, x[:1], workspace=x)
    p = [torch.zeros(4), torch.zeros(2, 3)]
    m3.adamw_table(p, p, p, p)
    for args in ((p, p[:1], p, p), (p, [v.half() for v in p], p, p), (p, p, [v.double() for v in p], p),
                 (p, p, p, p[::-1]), ([v.half() for v in p], p, p, p)):
        with pytest.raises(ValueError):
            m3.adamw_table(*args)
    with pytest.raises(ValueError):
        m3.adamw_table(p, p, p, p, scales=[torch.zeros(1, 2)] * 2)       # states not in 8 bits
    with pytest.raises(ValueError):
        m3.adamw_step(m3.adamw_table(p, p, p, p), step=1, lr=1.0, grad_scale=torch.zeros(2))


def test_binding_refuses_host_tensors():
    """Calls that are right but for lying in host memory."""
    x, A = torch.zeros(2, 5, 8, dtype=torch.bfloat16), -torch.ones(8)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    W, Wd = torch.zeros(12, 8, dtype=torch.bfloat16), torch.zeros(8, 12, dtype=torch.bfloat16)
    p, s = [torch.zeros(4)], torch.zeros(2, 1, 8)
    for call in (lambda: m3.glr_fwd(x, x, x, A, workspace=ws), lambda: m3.glr_bwd(x, x, x, A, s, x, workspace=ws),
                 lambda: m3.glr_step(torch.zeros(2, 8), x[:, 0], x[:, 0], x[:, 0], A),
                 lambda: m3.ffn_fwd(x, W, W, Wd, workspace=ws), lambda: m3.ffn_bwd(x, W, W, Wd, x, workspace=ws),
                 lambda: m3.adamw_step(m3.adamw_table(p, p, p, p), step=1, lr=1.0)):
        with pytest.raises(ValueError, match="of a GPU"):
            call()


@pytest.mark.parametrize("raw", [False, True])
def test_a_given_stream_orders_what_a_call_allocates(two_streams, raw):
    """With `stream` another than the current one, outputs, workspaces and their clearing
    are in the given stream's order (the kernels read the cleared workspace), and the
    outputs are kept for the caller's."""
    here, side, log = two_streams
    s = side.cuda_stream if raw else side
    x, A = torch.zeros(2, 5, 8, dtype=torch.bfloat16), -torch.ones(8)
    W, Wd = torch.zeros(12, 8, dtype=torch.bfloat16), torch.zeros(8, 12, dtype=torch.bfloat16)
    states, one = torch.zeros(2, 1, 8), torch.zeros(2, 8, dtype=torch.bfloat16)
    for call in (lambda: m3.glr_fwd(x, x, x, A, save_states=True, stream=s), lambda: m3.glr_bwd(x, x, x, A, states, x, stream=s),
                 lambda: m3.glr_step(torch.ones(2, 8), one, one, one, A, stream=s),
                 lambda: m3.ffn_fwd(x, W, W, Wd, stream=s), lambda: m3.ffn_bwd(x, W, W, Wd, x, stream=s)):
        log.clear()
        out = call()
        out = list(out.values()) if isinstance(out, dict) else list(out) if isinstance(out, tuple) else [out]
        ran = [e for e in log if e[0] != "kept for"]
        assert ran[-1][0].startswith("m3_") and len(ran) >= 2
        assert all(e[1] == side.cuda_stream and e[2] == side.cuda_stream for e in ran), ran
        assert sorted(e[2] for e in log if e[0] == "kept for") == sorted(t.data_ptr() for t in out)
        assert all(e[1] == here.cuda_stream for e in log if e[0] == "kept for")


def test_a_given_stream_with_everything_supplied(two_streams):
    """Nothing to allocate: the call goes straight to the given stream."""
    here, side, log = two_streams
    x, A, y, fs = torch.zeros(2, 5, 8), -torch.ones(8), torch.zeros(2, 5, 8), torch.zeros(2, 8)
    ws = torch.zeros(4096, dtype=torch.uint8)
    log.clear()
    m3.glr_fwd(x, x, x, A, out=(y, fs), workspace=ws, stream=side)
    m3.glr_step(fs, x[:, 0].contiguous(), x[:, 0].contiguous(), x[:, 0].contiguous(), A, y=y[:, 0].contiguous(), stream=side)
    m3.ffn_fwd(x, torch.ones(12, 8), torch.ones(12, 8), torch.ones(8, 12), out=y, workspace=ws, stream=side)
    assert [e for e in log if e[0].startswith("m3_")] == [(n, 2, 1) for n in ("m3_glr_fwd", "m3_glr_step", "m3_ffn_fwd")]
    assert not [e for e in log if e[0] in ("empty", "empty_like", "kept for")]


@pytest.mark.gpu
def test_binding_refuses_workspaces_and_scalars_elsewhere():
    x, A = torch.zeros(2, 5, 8, dtype=torch.bfloat16, device="cuda"), -torch.ones(8, device="cuda")
    W, Wd = x.new_zeros(12, 8), x.new_zeros(8, 12)
    for ws in (torch.zeros(1 << 26, dtype=torch.uint8), torch.zeros(1 << 24, device="cuda"),
               torch.zeros(1 << 27, dtype=torch.uint8, device="cuda")[::2]):
        for call in (lambda: m3.glr_fwd(x, x, x, A, workspace=ws), lambda: m3.ffn_fwd(x, W, W, Wd, workspace=ws),
                     lambda: m3.ffn_bwd(x, W, W, Wd, x, workspace=ws)):
            with pytest.raises(ValueError, match="workspace"):
                call()
    with pytest.raises(ValueError):
        m3.glr_fwd(x, x, x, A.cpu())
    p = [torch.zeros(4, device="cuda")]
    with pytest.raises(ValueError):
        m3.adamw_step(m3.adamw_table(p, p, p, p), step=1, lr=1.0, grad_scale=torch.ones(1))


def test_adamw_numbers_on_the_device(L):
    """t and lr on the device: their alignment is checked, the host's are not looked at."""
    _, p = plan(L, [tensor(n=0, p=None)])        # (nothing to do, nothing launched)

    def step(device_step=None, device_lr=None, table=None, pl=p, **kw):
        c = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, seed=0)
        c.update(kw)
        c = m3.M3AdamwConfig(*[c[k] for k in ("lr", "beta1", "beta2", "eps", "step", "seed")], device_step, device_lr)
        return L.m3_adamw_step(ctypes.byref(c), ctypes.byref(pl), table, None, None)
    assert step(device_step=FAKE + 4) == m3.M3_ERR_ALIGN and step(device_lr=FAKE + 4) == m3.M3_ERR_ALIGN
    assert step(device_step=FAKE, step=0) == m3.M3_OK and step(device_lr=FAKE, step=0) == m3.M3_ERR_SHAPE
    assert step(device_lr=FAKE, lr=float("nan")) == m3.M3_OK and step(device_step=FAKE, lr=float("nan")) == m3.M3_ERR_SHAPE


def test_ffn_room_for_any_weights(L):
    """Weights of whole rows that do not start on 16 bytes are refused where the workspace
    has no room for their copies; the room asked for is that of the three."""
    def call(d, weights, wsb):
        return L.m3_ffn_fwd(ctypes.byref(d), None, *weights, None, FAKE, wsb, None)
    d, none = ffn(), ffn(tokens=0)      # (no tokens: nothing to do, nothing launched)
    size = lambda d, what: L.m3_ffn_workspace_bytes(ctypes.byref(d), what)  # noqa: E731
    for what in (0, m3.M3_FFN_BACKWARD):
        assert size(d, what | m3.M3_FFN_ANY_WEIGHTS) - size(d, what) == 3 * 64 * 160 * 2
    assert size(d, 4) == 0
    odd = ffn(dmodel=65, x_stride=65, dff=161)                       # (copied anyway)
    assert size(odd, m3.M3_FFN_ANY_WEIGHTS) == size(odd, 0)
    room = size(none, m3.M3_FFN_ANY_WEIGHTS)
    for weights in ((FAKE + 2, FAKE, FAKE), (FAKE, FAKE + 8, FAKE), (FAKE, FAKE, FAKE + 14)):
        assert call(none, weights, room - 1) == m3.M3_ERR_ALIGN and call(none, weights, room) == m3.M3_OK
        assert call(none, [w + 1 for w in weights], room) == m3.M3_ERR_ALIGN
