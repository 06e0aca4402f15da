"""The classifier's loss with its gradients (ac_linear_ce_*) against a plain 64-bit implementation.

Tolerances. Products of bf16 values are exact in fp32; the tensor core adds D/16 groups of 16 of them to an fp32 sum, each
addition off by at most one unit in the last place of the running sum (2^-23), so a logit is off by at most about
(D/16 + 8) 2^-23 of the largest running sum, taken as twice the largest logit; exp and log add 4 units each. The gradients'
operand g is rounded to bf16 (2^-9 of each entry at most, 2^-9 / sqrt 3 in the mean square), after an fp16 rounding of 2^-12
where the logits' own pass left it, and each result once more: sqrt(2 / 3) 2^-9 = 1.6e-3 of the result's norm where the terms
of a sum are independent, 2 * 2^-9 = 3.9e-3 at worst."""
import math

import pytest

import __graft_entry__ as entry

pytestmark = pytest.mark.gpu

TOL_GRAD = 2 * 2.0 ** -9 + 2.0 ** -12


@pytest.fixture(scope="module")
def ac():
    entry.build()
    import paper_2409_11902_b200 as ac
    return ac


def make(T, V, D, bias, seed, ignored=0.2, spread=1.5):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    w = (torch.randn((V, D), generator=g, device="cuda") * spread / math.sqrt(D)).bfloat16()
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    h = (torch.randn((T, D), generator=g, device="cuda") + w[labels].float()).bfloat16()
    b = torch.randn((V,), generator=g, device="cuda").bfloat16() if bias else None
    if ignored and T > 1:
        labels[torch.rand((T,), generator=g, device="cuda") < ignored] = -100
    dloss = torch.rand((T,), generator=g, device="cuda") / T + 0.5 / T
    return h, w, b, labels, dloss


def plain(h, w, b, labels, dloss):
    import torch
    h, w = h.double(), w.double()
    x = h @ w.T if b is None else h @ w.T + b.double()
    V = w.shape[0]
    counts = (labels >= 0) & (labels < V)
    at = torch.where(counts, labels, 0)
    lse = torch.logsumexp(x, 1)
    loss = torch.where(counts, lse - x.gather(1, at[:, None])[:, 0], 0.0)
    p = torch.exp(x - lse[:, None])
    p[torch.arange(len(h), device=h.device), at] -= 1
    p = torch.where(counts[:, None], p * dloss.double()[:, None], 0.0)
    return dict(loss=loss, lse=lse, dh=p @ w, dw=p.T @ h, dbias=p.sum(0), top=float(x[x.isfinite()].abs().max()))


def run(ac, mode, h, w, b, labels, dloss, lse=None, nbytes=None, stream=None):
    import torch
    T, D = h.shape
    V = w.shape[0]
    d = ac.LinearCeDesc(T, V, D, bias=b is not None)
    nbytes = ac.ac_linear_ce_workspace_bytes(d) if nbytes is None else nbytes
    ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN wherever scratch is read before written
    nan = lambda *s, **k: torch.full(s, float("nan"), device="cuda", **k)  # noqa: E731
    o = dict(loss=nan(T), lse=nan(T) if lse is None else lse, dh=nan(T, D, dtype=torch.bfloat16),
             dw=nan(V, D, dtype=torch.bfloat16), dbias=nan(V, dtype=torch.bfloat16) if b is not None else None)
    if mode == "forward":
        ac.ac_linear_ce_forward(d, h, w, b, labels, o["loss"], o["lse"], ws, stream=stream)
    elif mode == "backward":
        ac.ac_linear_ce_backward(d, h, w, b, labels, o["lse"], dloss, o["dh"], o["dw"], o["dbias"], ws, stream=stream)
    else:
        ac.ac_linear_ce_step(d, h, w, b, labels, dloss, o["loss"], o["lse"], o["dh"], o["dw"], o["dbias"], ws, stream=stream)
    assert ac.ac_workspace_status(ws, stream) == (0, 0)
    return o


def tol_loss(D, top):
    return (D / 16 + 8) * 2.0 ** -23 * 2 * top + 16 * 2.0 ** -23 * max(top, 1.0)


def check_loss(o, want, D):
    tol = tol_loss(D, want["top"])
    assert float((o["lse"].double() - want["lse"]).abs().max()) <= tol
    assert float((o["loss"].double() - want["loss"]).abs().max()) <= 2 * tol


def check_grads(o, want, labels):
    V = want["dw"].shape[0]
    for k in ("dh", "dw", "dbias"):
        if o[k] is None:
            continue
        err = float((o[k].double() - want[k]).norm() / want[k].norm().clamp_min(1e-300))
        assert err <= TOL_GRAD, (k, err)
    dead = (labels < 0) | (labels >= V)
    assert bool((o["dh"][dead] == 0).all())


SIZES = [
    (1, 2, 8), (1, 1000, 512), (3, 1, 16), (7, 500, 100), (32, 1000, 512), (64, 129, 64), (129, 257, 72), (128, 1003, 8),
    (257, 4097, 264), (5, 70001, 24), (33, 515, 1), (31, 130, 13), (130, 1031, 1021),      # widths that are no multiple of 8
    (600, 6500, 96), (513, 10007, 520), (700, 9001, 333),                                  # tiles of CTA pairs
]


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("bias", [False, True])
def test_step_matches_the_definition(ac, T, V, D, bias):
    x = make(T, V, D, bias, seed=T + V + D)
    want = plain(*x)
    o = run(ac, "step", *x)
    check_loss(o, want, D)
    if V > 1:
        check_grads(o, want, x[3])
    else:       # one class: its probability is 1 and every gradient is 0
        assert float(o["dh"].float().abs().max()) <= 1e-6 and float(o["dw"].float().abs().max()) <= 1e-6


@pytest.mark.parametrize("T,V,D", [(1, 1000, 512), (129, 1003, 72), (31, 130, 13), (513, 10007, 520)])
def test_forward_and_backward_alone(ac, T, V, D):
    x = make(T, V, D, True, seed=5)
    want = plain(*x)
    f = run(ac, "forward", *x)
    check_loss(f, want, D)
    assert bool(f["dh"].isnan().all())
    b = run(ac, "backward", *x, lse=f["lse"].clone())
    check_grads(b, want, x[3])


@pytest.mark.parametrize("T,V,D", [(8200, 9001, 64), (8200, 9001, 20), (16500, 5000, 16)])
@pytest.mark.parametrize("mode", ["step", "backward"])
def test_pieces_give_the_same_as_one(ac, T, V, D, mode):
    """The least scratch (several pieces), a size between, and room for all classes."""
    x = make(T, V, D, True, seed=9)
    want = plain(*x)
    d = ac.LinearCeDesc(T, V, D, bias=True)
    least, ample = ac.ac_linear_ce_workspace_bytes_min(d), ac.ac_linear_ce_workspace_bytes(d)
    assert least < ample
    for nbytes in (least, (least + ample) // 2, ample):
        lse = None if mode == "step" else want["lse"].float()
        o = run(ac, mode, *x, lse=lse, nbytes=nbytes)
        if mode == "step":
            check_loss(o, want, D)
        check_grads(o, want, x[3])


def test_a_step_is_deterministic_and_independent_of_what_ran_before(ac):
    import torch
    x = make(300, 5003, 192, True, seed=3)
    a = run(ac, "step", *x)
    run(ac, "step", *make(300, 5003, 192, True, seed=4))
    b = run(ac, "step", *x)
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("floor", [float("-inf"), -3.3895313892515355e38])
def test_masked_classes_and_rows_that_do_not_count(ac, floor):
    import torch
    h, w, b, labels, dloss = make(200, 1003, 64, True, seed=11)
    off = torch.zeros(1003, dtype=torch.bool, device="cuda")
    off[100:400] = True
    off[torch.randint(0, 1003, (200,), device="cuda")] = True
    b = torch.where(off, floor, b.float()).bfloat16()
    labels = torch.where(labels >= 0, torch.where(off[labels.clamp(min=0)], 1003, labels), labels)     # outside: does not count
    want = plain(h, w, b, labels, dloss)
    o = run(ac, "step", h, w, b, labels, dloss)
    tol = tol_loss(64, 20.0)
    assert float((o["lse"].double() - want["lse"]).abs().max()) <= tol
    assert float((o["loss"].double() - want["loss"]).abs().max()) <= 2 * tol
    check_grads(o, want, labels)
    assert bool((o["dw"][off] == 0).all()) and bool((o["dbias"][off] == 0).all())
    # no row counts: everything is zero, even with NaN where the rows' weights stand
    none = torch.full_like(labels, -1)
    o = run(ac, "step", h, w, b, none, torch.full_like(dloss, float("nan")))
    for k in ("loss", "dh", "dw", "dbias"):
        assert bool((o[k] == 0).all()), k
    assert bool(o["lse"].isfinite().all())


def test_infinities_and_nan_stay_in_their_rows(ac):
    import torch
    h, w, b, labels, dloss = make(150, 700, 64, False, seed=12, ignored=0)
    h[3, 5] = float("nan")
    h[40, 7] = float("inf")
    o = run(ac, "step", h, w, b, labels, dloss)
    bad = torch.zeros(150, dtype=torch.bool, device="cuda")
    bad[[3, 40]] = True
    assert bool(o["loss"][bad].isnan().all()) and bool(o["loss"][~bad].isfinite().all())
    assert bool(o["dh"][~bad].isfinite().all())


def test_large_logits_do_not_overflow(ac):
    x = make(130, 900, 128, False, seed=13, spread=300.0)      # logits of several hundred
    want = plain(*x)
    o = run(ac, "step", *x)
    check_loss(o, want, 128)
    # p = exp(l - lse): an error of the logits of 2^-17 (a few hundred, 2^-23 each over the sums) is one of 1e-5 in p
    check_grads(o, want, x[3])


def test_gradients_match_differences_of_the_loss(ac):
    import torch
    h, w, b, labels, dloss = make(64, 601, 96, True, seed=14)
    o = run(ac, "step", h, w, b, labels, dloss)
    total = lambda h, w, b: float((plain(h, w, b, labels, dloss)["loss"] * dloss.double()).sum())  # noqa: E731
    g = torch.Generator("cuda").manual_seed(15)
    for i, k in enumerate(("dh", "dw", "dbias")):
        x = [h.double(), w.double(), b.double()]
        step = torch.randn(x[i].shape, generator=g, device="cuda", dtype=torch.float64)
        step = step + 2 * o[k].double() / o[k].double().norm() * step.norm()      # mostly along the gradient
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + 1e-5 * step, x[i] - 1e-5 * step
        slope = (total(*up) - total(*down)) / 2e-5
        assert abs(float((o[k].double() * step).sum()) - slope) <= 2 * TOL_GRAD * float(o[k].double().norm() * step.norm())


def test_another_stream(ac):
    import torch
    x = make(256, 1000, 256, True, seed=16)
    want = plain(*x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = run(ac, "step", *x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    check_loss(o, want, 256)
    check_grads(o, want, x[3])


def test_a_captured_step_replays(ac):
    import torch
    T, V, D = 96, 2000, 128
    h, w, b, labels, dloss = make(T, V, D, False, seed=17)
    d = ac.LinearCeDesc(T, V, D)
    ws = torch.empty(ac.ac_linear_ce_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    call = lambda: ac.ac_linear_ce_step(d, h, w, None, labels, dloss, loss, lse, dh, dw, None, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    h2, _, _, labels2, _ = make(T, V, D, False, seed=18)
    h.copy_(h2)
    labels.copy_(labels2)
    graph.replay()
    want = plain(h, w, b, labels, dloss)
    check_loss(dict(loss=loss, lse=lse), want, D)
    check_grads(dict(dh=dh, dw=dw, dbias=None), want, labels)
