"""Uncompressed embedding table on the GPU against the fp64 oracle.

Tolerances: a looked-up entry is one fp32 product (half a step of fp32) and,
in bf16, one more rounding.  A gradient entry sums m tokens in fp32: at most
m additions and the product with the scale, each off by half a step of a
value that the sum of the magnitudes bounds, then the rounding of its type.
"""
import numpy as np
import pytest

from oracle import dense_embed as OE
from paper_2405_14377_amd import comera as C
from tests.step_util import HALF, U, Guarded, dev, tdt, values, within

pytestmark = pytest.mark.gpu

CODE = {"f32": C.F32, "bf16": C.BF16}


def _ids(rng, n, V, kind):
    if kind == "same":
        return np.full(n, V - 1)
    if kind == "hot":
        return np.where(rng.random(n) < 0.5, 0, rng.integers(0, V, n))
    if kind == "neighbours":                  # a few ids that lie side by side
        return rng.integers(0, min(V, 5), n)
    return rng.integers(0, V, n)


def _dev_ids(ids):
    import torch
    return torch.from_numpy(np.asarray(ids, np.int64)).cuda()


def _backward(V, E, ids, dY, scale, pad, table="f32", act="f32", offset=0, ws=None, flag=None):
    import torch
    s = C.dense_embed_shape(V, E, CODE[table], CODE[act])
    out = Guarded((V, E), table, offset)
    ws = ws if ws is not None else torch.full((C.comera_dense_embed_workspace_bytes(s, len(ids)),), 0xA5,
                                              dtype=torch.uint8, device="cuda")
    C.comera_dense_embed_backward(s, _dev_ids(ids), len(ids), dev(dY, act, offset), scale, pad, out.t, ws, flag)
    return out


def _check_backward(got, V, ids, dY, scale, pad, table):
    scale = float(np.float32(scale))
    ref, mag = OE.backward(ids, dY, V, scale, pad), OE.backward(ids, np.abs(dY), V, abs(scale), pad)
    m = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
    within(got, ref, (m + 2) * U * mag + HALF[table] * np.abs(ref) * (1 + 1e-3) + 1e-38)


@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("V,E,n,offset", [(1, 1, 1, 0), (7, 3, 20, 1), (50, 8, 33, 0), (50, 9, 1, 3),
                                          (300, 100, 257, 0), (300, 128, 63, 0), (300, 129, 257, 1),
                                          (64, 256, 70, 0), (64, 257, 70, 3), (1000, 768, 130, 0), (33, 1001, 65, 1),
                                          (20, 4097, 9, 0)])
def test_forward(V, E, n, offset, table, act):
    rng = np.random.default_rng(V + E)
    T = values(rng.standard_normal((V, E)), table)
    ids = rng.integers(0, V, n)
    ids[-1] = 0
    s = C.dense_embed_shape(V, E, CODE[table], CODE[act])
    Y = Guarded((n, E), act, offset)
    scale = 27.7
    C.comera_dense_embed_forward(s, _dev_ids(ids), n, dev(T, table, offset), scale, Y.t)
    ref = OE.forward(ids, T, float(np.float32(scale)))
    within(Y.np(), ref, (U + (HALF[act] if act == "bf16" else 0)) * np.abs(ref) * (1 + 1e-3))


def test_forward_ids_out_of_range():
    import torch
    T = np.arange(12.0).reshape(4, 3)
    ids = np.array([3, -1, 4, 0, 2 ** 40, -2 ** 62])
    Y, flag = Guarded((6, 3), "f32"), torch.zeros(1, dtype=torch.int32, device="cuda")
    s = C.dense_embed_shape(4, 3)
    C.comera_dense_embed_forward(s, _dev_ids(ids[[0, 3]]), 2, dev(T), 2.0, Y.t, flag)
    assert flag.item() == 0
    C.comera_dense_embed_forward(s, _dev_ids(ids), 6, dev(T), 2.0, Y.t, flag)
    assert flag.item() == 1
    assert np.array_equal(Y.np(), OE.forward(ids, T, 2.0))


@pytest.mark.parametrize("kind", ["uniform", "hot", "same", "neighbours"])
@pytest.mark.parametrize("V,E,n", [(1, 1, 1), (3, 5, 40), (255, 8, 64), (256, 12, 65), (257, 64, 1000),
                                   (1000, 33, 2049), (4000, 96, 777), (300000, 2, 5000), (700001, 1, 300),
                                   # the last batch of one launch, the first of three; V beyond the one launch's
                                   (2000, 260, 1024), (2000, 260, 1025), (4194305, 1, 700), (5, 40, 3000),
                                   # the last batch in one part, the first in several; fewer ids than workgroups
                                   (257, 64, 24575), (257, 64, 24576), (20, 12, 30000), (70000, 4, 65537)])
def test_backward_sizes(V, E, n, kind):
    rng = np.random.default_rng(n)
    ids, dY = _ids(rng, n, V, kind), values(rng.standard_normal((n, E)), "f32")
    got = _backward(V, E, ids, dY, 0.5, -1)
    _check_backward(got.np(), V, ids, dY, 0.5, -1, "f32")


# one launch up to 256 tokens a row, its waves shared by one id; parts from 12288 tokens
@pytest.mark.parametrize("kind", ["uniform", "hot", "same"])
@pytest.mark.parametrize("V,E,n", [(1, 100, 17), (1, 768, 256), (1, 768, 257), (1, 3, 1024), (2, 768, 512),
                                   (2, 1001, 513), (3, 260, 700), (6, 2100, 1000), (5000, 768, 900), (1, 260, 12287),
                                   (1, 260, 12288), (4, 33, 12288), (2, 515, 16384), (2, 1, 16384), (3, 64, 40001),
                                   (17, 768, 2500)])
def test_backward_few_rows(V, E, n, kind):
    rng = np.random.default_rng(n + E)
    act = ("f32", "bf16")[n % 2]
    ids, dY = _ids(rng, n, V, kind), values(rng.standard_normal((n, E)), act)
    pad = (-1, V - 1)[E % 2]
    got = _backward(V, E, ids, dY, 0.5, pad, act=act, offset=n % 3)
    _check_backward(got.np(), V, ids, dY, 0.5, pad, "f32")


@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("V,E,n,offset", [(90, 768, 400, 0), (90, 1001, 400, 1), (40, 7, 200, 3), (31, 520, 3000, 0),
                                          (12, 2050, 37, 1)])
def test_backward_types(V, E, n, offset, table, act):
    rng = np.random.default_rng(E)
    ids, dY = _ids(rng, n, V, "hot"), values(0.01 * rng.standard_normal((n, E)), act)
    got = _backward(V, E, ids, dY, 27.7, 3, table, act, offset)
    _check_backward(got.np(), V, ids, dY, 27.7, 3, table)


def test_backward_pad_and_out_of_range():
    import torch
    rng = np.random.default_rng(5)
    V, E, n = 40, 16, 500
    ids = rng.integers(-3, V + 3, n)
    ids[100:300] = 7
    ids[5] = 2 ** 33 + 1           # its low 32 bits are a good id
    dY = values(rng.standard_normal((n, E)), "f32")
    for pad in (-1, 7, 0, V - 1):
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = _backward(V, E, ids, dY, 1.0, pad, flag=flag).np()
        _check_backward(got, V, ids, dY, 1.0, pad, "f32")
        assert flag.item() == 1
        if pad >= 0:
            assert not got[pad].any()
    flag.zero_()
    _backward(V, E, np.clip(ids, 0, V - 1), dY, 1.0, 7, flag=flag)
    assert flag.item() == 0
    assert not _backward(V, E, np.full(n, 7), dY, 1.0, 7).np().any()        # padding alone
    assert not _backward(V, E, np.full(n, -1), dY, 1.0, -1).np().any()      # no good id


def test_backward_without_tokens():
    assert not _backward(300, 5, np.zeros(0, np.int64), np.zeros((0, 5)), 1.0, -1, "bf16").np().any()


def test_backward_rows_with_infinities_stay_apart():
    V, E, n = 9, 32, 64
    ids = np.arange(n) % 8
    dY = np.ones((n, E))
    dY[3], dY[4, 5] = np.inf, np.nan
    got = _backward(V, E, ids, dY, 1.0, -1, act="bf16").t.cpu().numpy()
    assert np.isinf(got[3]).all() and np.isnan(got[4, 5]) and np.isfinite(np.delete(got[4], 5)).all()
    assert (got[[0, 1, 2, 5, 6, 7]] == 8).all() and not got[8].any()
    # an id that is padding takes nothing along
    assert not np.isnan(_backward(V, E, ids, dY, 1.0, 4, act="bf16").t.cpu().numpy()).any()


def test_backward_is_repeatable():
    rng = np.random.default_rng(6)
    V, E, n = 500, 130, 9000
    ids, dY = _ids(rng, n, V, "hot"), rng.standard_normal((n, E))
    a = _backward(V, E, ids, dY, 1.0, -1, act="bf16").np()
    assert all(np.array_equal(a, _backward(V, E, ids, dY, 1.0, -1, act="bf16").np()) for _ in range(3))


def test_large_offsets():
    """Entries behind 2^31 of the table, of Y and of dT."""
    import torch
    V, E, n = 70000, 32768, 40
    s = C.dense_embed_shape(V, E, C.BF16, C.BF16)
    T = torch.zeros((V, E), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 2, V - 1] * 10, device="cuda")
    rows = torch.randn((3, E), device="cuda").bfloat16()
    T[V - 1], T[0], T[V - 2] = rows[0], rows[1], rows[2]
    Y = torch.empty((n, E), dtype=torch.bfloat16, device="cuda")
    C.comera_dense_embed_forward(s, ids, n, T, 1.0, Y)
    assert torch.equal(Y, rows[[0, 1, 2, 0] * 10])
    T.fill_(5.0)
    ws = torch.empty(C.comera_dense_embed_workspace_bytes(s, n), dtype=torch.uint8, device="cuda")
    C.comera_dense_embed_backward(s, ids, n, torch.ones_like(Y), 1.0, -1, T, ws)
    assert (T[V - 1] == 20).all() and (T[V - 2] == 10).all() and (T[0] == 10).all()
    assert T[1:V - 2].count_nonzero().item() == 0
