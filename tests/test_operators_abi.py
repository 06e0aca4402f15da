"""Host-side checks of the loss and update operators: no GPU needed, every call returns before it touches CUDA."""
import ctypes
import dataclasses

import pytest

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def ac():
    entry.build()
    import paper_2409_11902_b200 as ac
    return ac


A = 0x10000      # 16-byte aligned, never dereferenced


def test_linear_ce_workspace(ac):
    d = ac.LinearCeDesc(8192, 131072, 4096)
    least, ample = ac.ac_linear_ce_workspace_bytes_min(d), ac.ac_linear_ce_workspace_bytes(d)
    stats, dh = 8 * 8192 * 131072 // 128, 4 * 8192 * 4096
    assert least < (64 << 20) + stats + dh + (1 << 20)          # a piece, the statistics, dh in fp32
    assert (2 << 30) <= ample < (2 << 30) + stats + (1 << 20)   # all of g: 8192 x 131072 in bf16
    huge = dataclasses.replace(d, tokens=1 << 17)
    assert ac.ac_linear_ce_workspace_bytes(huge) < (2 << 30) + 16 * stats + 16 * dh + (1 << 20)
    for bad in (dict(tokens=0), dict(classes=-1), dict(features=0), dict(dtype="f32")):
        b = dataclasses.replace(d, **bad)
        assert ac.ac_linear_ce_workspace_bytes(b) == 0 and ac.ac_linear_ce_workspace_bytes_min(b) == 0, bad
    assert ac.api.lib().ac_linear_ce_workspace_bytes(None) == 0


def test_linear_ce_refusals(ac):
    L, api = ac.api.lib(), ac.api
    big = 1 << 30

    def step(desc, bytes_=big, **kw):
        p = dict(h=A, w=A, bias=None, labels=A, dloss=A, loss=A, lse=A, dh=A, dw=A, dbias=None, workspace=A)
        p.update(kw)
        c = desc.c() if desc is not None else None
        return L.ac_linear_ce_step(ctypes.byref(c) if c else None, *p.values(), bytes_, None)

    d = ac.LinearCeDesc(32, 1000, 64)
    assert step(None) == api.AC_ERR_INVALID_ARG
    for k in ("h", "w", "labels", "dloss", "loss", "lse", "dh", "dw", "workspace"):
        assert step(d, **{k: None}) == api.AC_ERR_INVALID_ARG, k
        assert step(d, **{k: A + 8}) == api.AC_ERR_MISALIGNED, k
    b = dataclasses.replace(d, bias=True)
    assert step(d, bias=A, dbias=A) == api.AC_ERR_INVALID_ARG       # a bias that the descriptor does not name
    assert step(b) == api.AC_ERR_INVALID_ARG
    assert step(b, bias=A) == api.AC_ERR_INVALID_ARG
    assert step(b, bias=A, dbias=A + 2) == api.AC_ERR_MISALIGNED
    assert step(dataclasses.replace(d, tokens=0)) == api.AC_ERR_INVALID_ARG
    assert step(dataclasses.replace(d, dtype="f32")) == api.AC_ERR_UNSUPPORTED
    assert step(d, bytes_=ac.ac_linear_ce_workspace_bytes_min(d) - 1) == api.AC_ERR_WORKSPACE_TOO_SMALL
    c = d.c()
    c.dtype = 9
    assert L.ac_linear_ce_forward(ctypes.byref(c), A, A, None, A, A, A, A, big, None) == api.AC_ERR_INVALID_ARG
    c = d.c()
    c.has_bias = 2
    assert L.ac_linear_ce_forward(ctypes.byref(c), A, A, None, A, A, A, A, big, None) == api.AC_ERR_INVALID_ARG
    c = d.c()
    assert L.ac_linear_ce_forward(ctypes.byref(c), A, A, None, A, None, A, A, big, None) == api.AC_ERR_INVALID_ARG
    assert L.ac_linear_ce_forward(ctypes.byref(c), A, A, None, A, A, A, A, 100, None) == api.AC_ERR_WORKSPACE_TOO_SMALL
    assert L.ac_linear_ce_backward(ctypes.byref(c), A, A, None, A, None, A, A, A, None, A, big, None) == api.AC_ERR_INVALID_ARG
    assert L.ac_linear_ce_backward(ctypes.byref(c), A, A, None, A, A, A, A, A, None, A, 100, None) == api.AC_ERR_WORKSPACE_TOO_SMALL


def test_muon_refusals(ac):
    L, api = ac.api.lib(), ac.api
    d = ac.MuonDesc(64, 576)
    need = ac.ac_muon_workspace_bytes(d)
    assert 256 < need < 64 * 576 * 16

    def call(desc, bytes_=need, **kw):
        p = dict(grad=A, momentum_in=A, momentum_out=A, update=A, workspace=A)
        p.update(kw)
        c = desc.c() if desc is not None else None
        return L.ac_muon_update(ctypes.byref(c) if c else None, *p.values(), bytes_, None)

    assert call(None) == api.AC_ERR_INVALID_ARG
    for k in ("grad", "update", "workspace", "momentum_in", "momentum_out"):       # one momentum without the other, too
        assert call(d, **{k: None}) == api.AC_ERR_INVALID_ARG, k
        assert call(d, **{k: A + 4}) == api.AC_ERR_MISALIGNED, k
    assert call(d, bytes_=need - 1) == api.AC_ERR_WORKSPACE_TOO_SMALL
    for bad in (dict(rows=0), dict(cols=-3), dict(batch=0), dict(batch=70000), dict(steps=-1), dict(momentum=float("nan")),
                dict(scale=float("inf")), dict(eps=-1.0), dict(coefficients=(1.0, float("nan"), 0.0)), dict(rows=1 << 30, cols=1 << 30)):
        b = dataclasses.replace(d, **bad)
        assert ac.ac_muon_workspace_bytes(b) == 0, bad
        assert call(b) == api.AC_ERR_INVALID_ARG, bad
    c = d.c()
    c.dtype = 5
    assert L.ac_muon_workspace_bytes(ctypes.byref(c)) == 0


def test_bindings_raise(ac):
    d = ac.MuonDesc(8, 8)
    with pytest.raises(ac.AcError) as e:
        ac.ac_muon_update(d, None, None, None, A, A, 1 << 20, stream=0)
    assert e.value.status == ac.api.AC_ERR_INVALID_ARG
    with pytest.raises(ac.AcError):
        ac.ac_linear_ce_forward(ac.LinearCeDesc(8, 8, 8), A, A, None, A, None, A, A, 1 << 20, stream=0)


def test_every_call_accepts_the_least_workspace_and_all_above(ac):
    """Random problems: the least size never exceeds the ample one, and no call refuses a size from there on."""
    import math
    import random
    L, api, rng = ac.api.lib(), ac.api, random.Random(7)
    size = lambda top: int(math.exp(rng.uniform(0, math.log(top))))  # noqa: E731
    for _ in range(1500):
        d = ac.LinearCeDesc(size(70000), size(300000), size(9000), bias=rng.random() < 0.5)
        c = d.c()
        b = A if d.bias else None
        least, ample = ac.ac_linear_ce_workspace_bytes_min(d), ac.ac_linear_ce_workspace_bytes(d)
        assert 0 < least <= ample, d
        if api.torch.cuda.is_available():
            continue        # the addresses below are not memory: without a GPU the calls end at the first launch
        assert L.ac_linear_ce_forward(ctypes.byref(c), A, A, b, A, A, A, A, least, None) == api.AC_ERR_CUDA, d
        for n in (least, ample, rng.randint(least, ample)):
            assert L.ac_linear_ce_step(ctypes.byref(c), A, A, b, A, A, A, A, A, A, b, A, n, None) == api.AC_ERR_CUDA, (d, n)
            assert L.ac_linear_ce_backward(ctypes.byref(c), A, A, b, A, A, A, A, A, b, A, n, None) == api.AC_ERR_CUDA, (d, n)
