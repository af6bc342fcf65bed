"""What the calls around the layers promise beyond one call: workspaces of a
longest batch, a long list's table, raw addresses (no GPU: launch check mode,
placeholder addresses)."""
import pytest

from paper_2405_14377_amd import comera as C

FAKE = 1 << 40


@pytest.fixture
def checked():
    C.comera_debug_launch_check(True)
    yield
    C.comera_debug_launch_check(False)


# token counts around every change of the table gradient's form, for tables of more than four rows and of fewer
COUNTS = (0, 1, 100, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 2000, 12287, 12288, 12289, 24575, 24576, 24577,
          32767, 32768, 32769, 60000, 131072)


@pytest.mark.parametrize("V,E", [(1, 8), (2, 64), (4, 16), (5, 3), (100, 8), (2000, 640), (32768, 768), (70000, 4),
                                 (600000, 1), (4194304, 2), (4194305, 2)])
def test_embed_workspace_of_the_longest_batch(checked, V, E):
    """A workspace for n tokens serves every batch of up to n."""
    lib = C.load()
    s = C.dense_embed_shape(V, E, C.F32, C.BF16)
    sizes = [C.comera_dense_embed_workspace_bytes(s, n) for n in COUNTS]
    assert sizes == sorted(sizes)
    for i, most in enumerate(sizes):
        for n in COUNTS[:i + 1]:
            assert lib.comera_dense_embed_backward(s, FAKE, n, FAKE, 1.0, -1, FAKE, FAKE, most, None, 0) == C.OK, n


@pytest.mark.parametrize("width", [1, 8, 128, 256, 768, 1000, 4096, 5000, 8192])
def test_norm_workspace_of_the_longest_batch(width):
    s = C.block_norm_shape(width, pre=C.NORM_LAYER)
    sizes = [C.comera_block_norm_workspace_bytes(s, b) for b in range(3000)]
    assert sizes == sorted(sizes)


class OnDevice:
    """Host tensors that say they are on device 0, streams by their handles, and what a table was recorded on."""

    def __init__(self, monkeypatch, current=7):
        import torch
        self.recorded = []
        outer = self

        class Tensor(torch.Tensor):
            def get_device(self):
                return 0

            def record_stream(self, stream):
                outer.recorded.append(stream)

        class Current:
            cuda_stream = current

            def synchronize(self):
                pass

        empty = torch.empty
        self.tensor = lambda *a, **k: empty(*a, **{**k, "device": "cpu"}).as_subclass(Tensor)
        monkeypatch.setattr(torch, "empty", self.tensor)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Current())
        monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: "default")
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, *a: handle)
        monkeypatch.setattr(C, "_stream", lambda s: current if s is None else s)


def test_a_plans_table_is_recorded_on_every_stream(checked, monkeypatch):
    """A dropped plan's table waits for calls on other streams than the one it was made on."""
    d = OnDevice(monkeypatch)
    for count, table in ((120, False), (121, True)):
        plan = C.GradPlan([d.tensor(4) for _ in range(count)])
        assert (plan.table is not None) == table
        ws = d.tensor(plan.workspace_bytes // 4)
        norm = d.tensor(1)
        C.comera_grad_clip(plan.handle, 1.0, 1.0, norm, None, ws)             # the stream that made it
        C.comera_grad_clip(plan.handle, 1.0, 1.0, norm, None, ws, stream=21)
        C.comera_grad_clip(plan.handle, 1.0, 1.0, norm, None, ws, stream=21)
        C.comera_grad_norm(plan.handle, 1.0, norm, None, ws, stream=0)
        C.comera_grad_norm(plan.handle, 1.0, norm, None, ws, stream=22)
        assert d.recorded == ([21, "default", 22] if table else [])
        handle = plan.handle
        assert (handle in C._tables) == table
        del plan
        assert handle not in C._tables


WITHOUT_TORCH = """
import sys
sys.modules["torch"] = None               # an import of it fails
from paper_2405_14377_amd import comera as C
C.comera_debug_launch_check(True)
at = [(1 << 40) + (i << 36) for i in range(20)]
s = C.dense_embed_shape(100, 8, C.F32, C.BF16)
C.comera_dense_embed_forward(s, at[0], 4, at[1], 1.0, at[2], at[3], stream=0)
n = C.block_norm_shape(64, C.F32, C.BF16, C.NORM_LAYER, C.NORM_LAYER, C.GATE_TOKEN)
C.comera_block_norm_forward(n, 4, *at[:9], stream=0)
C.comera_block_norm_backward(n, 4, *at[:11], None, None, None, None, None, stream=0)
try:
    C.comera_dense_embed_forward(s, at[0], 4, at[1], 1.0, at[2])
except ImportError as e:
    assert "pass a stream" in str(e)
else:
    raise AssertionError("a current stream without torch")
plan = C.GradPlan([])
assert plan.table is None
p = C.comera_grad_plan((C.comera_grad_tensor * 1)((at[0], None, 100, C.BF16, 0)), 1)
"""


def _process(code):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr


def test_addresses_without_torch():
    """Raw addresses and a stream need no torch."""
    _process(WITHOUT_TORCH)


RAW_WORKSPACES = """
from paper_2405_14377_amd import comera as C
C.comera_debug_launch_check(True)
at = [(1 << 40) + (i << 36) for i in range(40)]
W = 1 << 34
many = (C.comera_grad_tensor * 200)(*[(at[0] + 64 * i, None, 16, C.F32, 0) for i in range(200)])
p = C.comera_grad_plan(many, 200)
s, n = C.dense_embed_shape(100, 8), C.block_norm_shape(64, pre=C.NORM_RMS)


def calls(ws, table):
    yield lambda: C.comera_dense_embed_backward(s, at[0], 4, at[1], 1.0, -1, at[2], ws, stream=0)
    yield lambda: C.comera_block_norm_backward(n, 4, at[0], None, None, None, None, at[1], at[2], at[3], at[4], None,
                                               None, None, None, at[5], None, ws, stream=0)
    yield lambda: C.comera_grad_plan_set_table(p, table, stream=0)
    yield lambda: C.comera_grad_norm(p, 1.0, at[1], None, ws, stream=0)
    yield lambda: C.comera_grad_clip(p, 1.0, 1.0, at[1], None, ws, stream=0)


for call in calls((at[6], W), (at[7], C.comera_grad_table_bytes(p))):
    assert call() == C.OK
# too short, none, and an address without its bytes
for ws in ((at[6], 8), None, at[6]):
    for i, call in enumerate(calls(ws, ws)):
        try:
            call()
        except C.ComeraError as e:
            assert e.status == C.ERR_WORKSPACE, e
        else:
            assert ws is None and i == 2          # no table: allowed
"""


def test_raw_workspaces():
    """A workspace or a table at a raw address comes with its bytes, with torch or without."""
    _process(RAW_WORKSPACES)
    _process("import sys\nsys.modules['torch'] = None\n" + RAW_WORKSPACES)
