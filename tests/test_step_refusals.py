"""What the operators around the layers refuse, on the host, and that their
launches fit the device at every size that they take (no GPU: launch check
mode, placeholder addresses)."""
import math

import pytest

from paper_2405_14377_amd import comera as C

FAKE = 1 << 40


@pytest.fixture
def checked():
    C.comera_debug_launch_check(True)
    yield
    log = C.comera_debug_launch_log()
    C.comera_debug_launch_check(False)
    assert not [x for x in log if not x["ok"]]
    # a launch counts its threads in 32 bits, and these kernels ask for no more LDS than any kernel may have
    for x in log:
        g, b = x["grid"], x["block"]
        assert g[0] * b[0] * g[1] * b[1] * g[2] * b[2] < 2 ** 32, x
        assert x["lds"] <= 64 * 1024, x


def _addr(i):
    return FAKE + (i << 36)


def test_embed_refusals(checked):
    lib = C.load()
    s, W = C.dense_embed_shape(100, 8), 1 << 30

    def fwd(s=s, ids=FAKE, n=4, T=FAKE, scale=1.0, Y=FAKE):
        return lib.comera_dense_embed_forward(s, ids, n, T, scale, Y, None, 0)

    def bwd(s=s, ids=FAKE, n=4, dY=FAKE, scale=1.0, pad=-1, dT=FAKE, ws=FAKE, w=W):
        return lib.comera_dense_embed_backward(s, ids, n, dY, scale, pad, dT, ws, w, None, 0)

    assert fwd() == C.OK and bwd() == C.OK
    bad = [C.dense_embed_shape(*x) for x in ((0, 8), (8, 0), (8, 8, 2), (8, 8, 0, -1))]
    for call in (fwd, bwd):
        for b in bad:
            assert call(s=b) == C.ERR_INVALID_ARG
        assert call(n=-1) == C.ERR_INVALID_ARG and call(n=2 ** 31 - 1) == C.ERR_INVALID_ARG
        assert call(ids=None) == C.ERR_INVALID_ARG
        assert call(scale=math.inf) == C.ERR_INVALID_ARG and call(scale=math.nan) == C.ERR_INVALID_ARG
        assert call(s=C.dense_embed_shape(2 ** 31 - 1, 1)) == C.ERR_UNSUPPORTED
        assert call(s=C.dense_embed_shape(1, 2 ** 31 - 1)) == C.ERR_UNSUPPORTED
    assert fwd(T=None) == C.ERR_INVALID_ARG and fwd(Y=None) == C.ERR_INVALID_ARG
    assert bwd(dY=None) == C.ERR_INVALID_ARG and bwd(dT=None) == C.ERR_INVALID_ARG
    assert bwd(pad=-2) == C.ERR_INVALID_ARG and bwd(pad=100) == C.ERR_INVALID_ARG and bwd(pad=99) == C.OK
    need = C.comera_dense_embed_workspace_bytes(s, 4)
    assert bwd(ws=None) == C.ERR_WORKSPACE and bwd(w=need - 1) == C.ERR_WORKSPACE and bwd(w=need) == C.OK
    assert bwd(ws=FAKE + 8) == C.ERR_WORKSPACE
    assert all(C.comera_dense_embed_workspace_bytes(b, 4) == 0 for b in bad)
    assert C.comera_dense_embed_workspace_bytes(s, -1) == 0
    # no tokens: nothing to read; the gradient is still written
    assert fwd(n=0, ids=None, T=None, Y=None) == C.OK
    assert bwd(n=0, ids=None, dY=None) == C.OK and bwd(n=0, ids=None, dY=None, dT=None) == C.ERR_INVALID_ARG


@pytest.mark.parametrize("V", [1, 2, 255, 256, 257, 524288, 524289, 2 ** 30, 2 ** 30 + 1, 2 ** 31 - 2])
@pytest.mark.parametrize("E", [1, 3, 4, 7, 8, 1001, 2 ** 20])
def test_embed_launches(checked, V, E):
    lib = C.load()
    for n in (0, 1, 63, 512, 513, 65537, 2 ** 31 - 2):
        for table in (C.F32, C.BF16):
            s = C.dense_embed_shape(V, E, table, C.BF16)
            assert lib.comera_dense_embed_forward(s, FAKE, n, FAKE, 1.0, FAKE, None, 0) == C.OK
            ws = C.comera_dense_embed_workspace_bytes(s, n)
            assert (ws > 0) == (V <= 2 ** 30)
            want = C.OK if V <= 2 ** 30 else C.ERR_UNSUPPORTED
            assert lib.comera_dense_embed_backward(s, FAKE, n, FAKE, 1.0, -1, FAKE, FAKE, ws, None, 0) == want


def _norm_calls(**k):
    """(forward, backward) with every pointer of a full block, some replaced."""
    lib = C.load()
    shape = k.pop("s", None) or C.block_norm_shape(64, C.F32, C.BF16, C.NORM_LAYER, C.NORM_LAYER, C.GATE_CHANNEL)
    names = ("X", "F", "post_w", "post_b", "gate", "pre_w", "pre_b", "Xn", "H", "dXn", "dH", "dX", "dF", "dgate",
             "dpost_w", "dpost_b", "dpre_w", "dpre_b", "ws")
    a = {n: _addr(i) for i, n in enumerate(names)}
    a.update(b=10, w=1 << 32)
    a.update(k)
    f = lib.comera_block_norm_forward(shape, a["b"], a["X"], a["F"], a["post_w"], a["post_b"], a["gate"], a["pre_w"],
                                      a["pre_b"], a["Xn"], a["H"], 0)
    g = lib.comera_block_norm_backward(shape, a["b"], a["Xn"], a["F"], a["post_w"], a["post_b"], a["gate"], a["pre_w"],
                                       a["dXn"], a["dH"], a["dX"], a["dF"], a["dgate"], a["dpost_w"], a["dpost_b"],
                                       a["dpre_w"], a["dpre_b"], a["ws"], a["w"], 0)
    return f, g


def test_norm_refusals(checked):
    N, R, L = C.NORM_NONE, C.NORM_RMS, C.NORM_LAYER
    bad, ok, ws = C.ERR_INVALID_ARG, C.OK, C.ERR_WORKSPACE
    assert _norm_calls() == (ok, ok)
    shape = C.block_norm_shape
    for s in (shape(0), shape(64, 2), shape(64, 0, 2), shape(64, post=3), shape(64, pre=-1), shape(64, gate=3),
              shape(64, eps=0.0), shape(64, eps=-1.0), shape(64, eps=math.nan), shape(64, res_scale=math.inf),
              shape(64, branch_scale=math.nan)):
        assert _norm_calls(s=s) == (bad, bad)
        assert C.comera_block_norm_workspace_bytes(s, 4) == 0
    for s in (shape(8193), shape(64, C.BF16, C.F32)):
        assert _norm_calls(s=s) == (C.ERR_UNSUPPORTED,) * 2
        assert C.comera_block_norm_workspace_bytes(s, 4) == 0
    assert _norm_calls(b=-1) == (bad, bad)
    assert _norm_calls(X=None)[0] == bad and _norm_calls(H=None)[0] == bad and _norm_calls(gate=None) == (bad, bad)
    assert _norm_calls(Xn=None) == (ok, bad)                     # dH is given: the backward reads Xn
    assert _norm_calls(Xn=None, dH=None)[1] == ok
    assert _norm_calls(dXn=None, dH=None)[1] == bad and _norm_calls(dXn=None)[1] == ok
    # no block before: nothing of one is passed
    assert _norm_calls(F=None) == (bad, bad)
    none = dict(F=None, post_w=None, post_b=None, gate=None, dF=None, dgate=None, dpost_w=None, dpost_b=None)
    assert _norm_calls(**none) == (bad, ok)                      # Xn would be X
    assert _norm_calls(**none, Xn=None)[0] == ok
    for extra in ("dF", "dgate", "dpost_w", "dpost_b", "post_w", "gate"):
        assert _norm_calls(**{**none, extra: FAKE})[1] == bad
    # what the shape rules out
    s = shape(64, post=N, pre=R, gate=C.GATE_CHANNEL)
    off = dict(post_w=None, post_b=None, dpost_w=None, dpost_b=None)
    assert _norm_calls(s=s, **off) == (ok, ok)
    for extra in off:
        assert bad in _norm_calls(s=s, **{**off, extra: FAKE})
    s = shape(64, post=R, pre=N, gate=C.GATE_NONE)
    off = dict(pre_w=None, pre_b=None, H=None, dH=None, dpre_w=None, dpre_b=None, gate=None, dgate=None)
    assert _norm_calls(s=s, **off) == (ok, ok)
    for extra in off:
        assert bad in _norm_calls(s=s, **{**off, extra: FAKE})
    # the workspace, needed only for the parameters' gradients
    need = C.comera_block_norm_workspace_bytes(shape(64), 10)
    assert _norm_calls(ws=None)[1] == ws and _norm_calls(w=need - 1)[1] == ws and _norm_calls(w=need)[1] == ok
    assert _norm_calls(ws=FAKE + 8)[1] == ws
    assert _norm_calls(ws=None, w=0, dgate=None, dpost_w=None, dpost_b=None, dpre_w=None, dpre_b=None)[1] == ok
    # empty batches
    assert _norm_calls(b=0, X=None, F=None, gate=None, Xn=None, H=None, dXn=None, dH=None, ws=None, w=0) == (ok, ok)


def test_norm_launches(checked):
    for width in (1, 7, 8, 127, 128, 129, 256, 257, 511, 512, 513, 768, 1024, 1025, 1537, 4096, 6144, 6145, 8192):
        for b in (1, 3, 4, 257, 1025, 70000, 2 ** 33):
            for s in (C.block_norm_shape(width, C.F32, C.F32, C.NORM_LAYER, C.NORM_LAYER, C.GATE_TOKEN),
                      C.block_norm_shape(width, C.BF16, C.BF16, C.NORM_RMS, C.NORM_RMS, C.GATE_CHANNEL)):
                assert _norm_calls(s=s, b=b, w=C.comera_block_norm_workspace_bytes(s, b)) == (C.OK, C.OK)
                assert _norm_calls(s=s, b=b, post_b=None, dpost_b=None, dpre_b=None) == (C.OK, C.OK)


def _plan(entries):
    arr = (C.comera_grad_tensor * max(1, len(entries)))()
    for i, (g, out, n, dtype) in enumerate(entries):
        arr[i] = C.comera_grad_tensor(g, out, n, dtype, 0)
    return C.comera_grad_plan(arr, len(entries), raise_on_error=False)


def test_grad_refusals(checked):
    lib = C.load()
    bad = C.ERR_INVALID_ARG
    st, p = _plan([(FAKE, None, 100, 0), (_addr(1), _addr(2), 100, 1)])
    assert st == C.OK
    need = C.comera_grad_workspace_bytes(p)
    W = 1 << 20

    def norm(p=p, scale=1.0, out=FAKE, flag=FAKE, ws=FAKE, w=W):
        return lib.comera_grad_norm(p, scale, out, flag, ws, w, 0)

    def clip(p=p, scale=1.0, out=FAKE, flag=FAKE, ws=FAKE, w=W, most=1.0):
        return lib.comera_grad_clip(p, scale, most, out, flag, ws, w, 0)

    for call in (norm, clip):
        assert call() == C.OK and call(w=need) == C.OK and call(flag=None) == C.OK and call(out=None) == C.OK
        assert call(p=None) == bad
        for scale in (0.0, -1.0, math.inf, math.nan):
            assert call(scale=scale) == bad
        assert call(ws=None) == C.ERR_WORKSPACE and call(w=need - 1) == C.ERR_WORKSPACE
        assert call(ws=FAKE + 8) == C.ERR_WORKSPACE
    assert norm(out=None, flag=None) == bad and clip(out=None, flag=None) == C.OK
    assert clip(most=-1.0) == bad and clip(most=math.nan) == bad and clip(most=math.inf) == C.OK
    C.comera_grad_plan_destroy(p)
    assert C.comera_grad_workspace_bytes(None) == 0
    assert lib.comera_grad_plan(None, 0, None) == bad
    assert lib.comera_grad_plan_set_table(None, FAKE, 1 << 20, 0) == bad and C.comera_grad_table_bytes(None) == 0
    for e in ([(None, None, 4, 0)], [(FAKE, None, -1, 0)], [(FAKE, None, 4, 2)], [(FAKE + 2, None, 4, 0)],
              [(FAKE, FAKE + 1025, 4, 1)], [(FAKE, None, 1 << 42, 0)],
              [(FAKE, None, 4, 0), (FAKE, None, 4, 0)],                       # the same tensor twice
              [(FAKE, None, 4, 0), (FAKE + 12, None, 4, 0)],                  # overlapping inputs
              [(FAKE, FAKE + 8, 4, 0)],                                       # an output over its own input, shifted
              [(FAKE, _addr(1), 4, 0), (_addr(2), _addr(1) + 4, 4, 0)],       # overlapping outputs
              [(FAKE, _addr(1), 4, 0), (_addr(1), None, 4, 0)]):              # an output over another input
        st, p = _plan(e)
        assert st == bad and not p, e
    # neighbours do not overlap, empty tensors are passed over
    st, p = _plan([(FAKE, None, 4, 0), (FAKE + 16, None, 4, 0), (None, None, 0, 0), (FAKE, None, 0, 1)])
    assert st == C.OK
    C.comera_grad_plan_destroy(p)


def test_grad_launches(checked):
    lib = C.load()
    for sizes in ([], [1], [1] * 500, [1 << 33], [1 << 41, 5], [8192] * 120, [8193] * 121, [10 ** 7] + [30] * 1000):
        entries, at = [], FAKE
        for i, n in enumerate(sizes):
            entries.append((at, None, n, i % 2))
            at += n * 4
        st, p = _plan(entries)
        assert st == C.OK
        w = C.comera_grad_workspace_bytes(p)
        assert lib.comera_grad_clip(p, 1.0, 1.0, FAKE, FAKE, FAKE, w, 0) == C.OK
        assert lib.comera_grad_norm(p, 1.0, FAKE, FAKE, FAKE, w, 0) == C.OK
        # a long list's table: one launch where there were several
        need = C.comera_grad_table_bytes(p)
        assert (need > 0) == (len(sizes) > 120)
        set_table = lib.comera_grad_plan_set_table
        assert set_table(p, None, 0, 0) == C.OK and set_table(p, FAKE, need, 0) == C.OK
        if need:
            assert set_table(p, FAKE, need - 1, 0) == C.ERR_WORKSPACE
            assert set_table(p, FAKE + 4, need, 0) == C.ERR_WORKSPACE
            before = C.comera_debug_launch_log()
            assert lib.comera_grad_clip(p, 1.0, 1.0, FAKE, FAKE, FAKE, w, 0) == C.OK
            without = len(C.comera_debug_launch_log()) - len(before)          # a refused table is none
            assert set_table(p, FAKE, need, 0) == C.OK
            before = C.comera_debug_launch_log()
            assert lib.comera_grad_clip(p, 1.0, 1.0, FAKE, FAKE, FAKE, w, 0) == C.OK
            assert len(C.comera_debug_launch_log()) - len(before) == 2 < without
        C.comera_grad_plan_destroy(p)


def test_tensor_checks():
    """What the binding refuses of tensors: host memory, another device, another type, strides, too few entries."""
    import torch
    s = C.dense_embed_shape(4, 3)
    T, ids = torch.zeros(4, 3), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(C.ComeraError) as e:
        C.comera_dense_embed_forward(s, ids, 2, T, 1.0, T, stream=0)
    assert e.value.status == C.ERR_INVALID_ARG and "host memory" in str(e.value)
    with pytest.raises(C.ComeraError):
        C.GradPlan([torch.zeros(3)])
    with pytest.raises(C.ComeraError):
        C.GradPlan([torch.zeros(3, dtype=torch.float16)])
    with pytest.raises(C.ComeraError):
        C.GradPlan([], [None])

    class Fake(torch.Tensor):
        """A host tensor that says it is on the current device."""
        def get_device(self):
            return 0

    def checked(t, dtype, n):
        assert C._taken("here", (t, dtype, n)) == [t if t is None or isinstance(t, int) else t.data_ptr()]

    from unittest import mock
    t = torch.zeros(4, 3).as_subclass(Fake)
    with mock.patch("torch.cuda.current_device", return_value=0):
        checked(t, torch.float32, 12)
        checked(None, torch.float32, 12)
        checked(FAKE, torch.float32, 12)
        for bad in ((t, torch.bfloat16, 12), (t, torch.float32, 13), (t.t(), torch.float32, 12)):
            with pytest.raises(C.ComeraError):
                checked(*bad)
    with mock.patch("torch.cuda.current_device", return_value=1):
        with pytest.raises(C.ComeraError, match="device"):
            checked(t, torch.float32, 12)
