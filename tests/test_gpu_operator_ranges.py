"""The loss and the update at the edges of their kernels' ranges: sizes on both sides of each choice of kernel and tile,
batches and matrices whose offsets pass 2^31 elements, extreme weights and scales. References and tolerances are those of
test_gpu_linear_ce.py and test_gpu_muon.py."""
import math

import pytest

import __graft_entry__ as entry
import test_gpu_linear_ce as ce
import test_gpu_muon as mu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ac():
    entry.build()
    import paper_2409_11902_b200 as ac
    return ac


# the on-chip kernel's last sizes and the first beyond them, few and many slabs per CTA, odd column counts (scalar loads)
ONCHIP = [(1, 32, 2560), (1, 32, 2561), (2, 2560, 31), (1, 33, 1344), (1, 33, 1345), (1, 1344, 64), (1, 64, 1349), (1, 65, 64),
          (3, 7, 2003), (2, 2001, 5), (200, 48, 96), (1, 64, 64), (1, 64, 65)]
# split tiles, slices, half of the tiles mirrored, tiles of pairs, each with its neighbours
LARGE = [(1, 96, 20000), (8, 2364, 35), (5, 1083, 321), (1, 771, 6000), (2, 130, 9000), (1, 1024, 1024), (1, 4200, 4100), (2, 2048, 2304),
         (12, 384, 384), (1, 5000, 700)]


@pytest.mark.parametrize("b,m,n", ONCHIP + LARGE)
def test_update_on_both_sides_of_each_choice(ac, b, m, n):
    grad, v = mu.matrix("noise", b, m, n, 21), 3 * mu.matrix("noise", b, m, n, 22)
    scale = math.sqrt(max(1.0, m / n))
    want_v, want = mu.plain(grad, v, 0.95, True, 5, scale, 1e-7)
    got_v, got = mu.run(ac, grad, v, momentum=0.95, scale=scale)
    assert float((got_v.double() - want_v).abs().max()) <= 2.0 ** -22 * float(want_v.abs().max())
    mu.check(got, want)


def test_a_batch_of_small_matrices_past_two_to_the_31(ac):
    """Each matrix is updated by itself: the last of a batch of 2.2e9 elements equals the same matrix alone, bit for bit."""
    import torch
    b, m, n = 34000, 64, 1024
    assert b * m * n > 1 << 31
    last = mu.matrix("noise", 1, m, n, 23).bfloat16()
    grad = torch.empty((b, m, n), dtype=torch.bfloat16, device="cuda")
    grad[:] = last
    grad[0] = 0
    grad[1:17000:1000] *= 2
    alone = mu.run(ac, last, None, momentum=0.0)[1][0]
    got = mu.run(ac, grad, None, momentum=0.0)[1]
    assert bool((got[0] == 0).all())
    assert torch.equal(got[-1], alone) and torch.equal(got[17001], alone) and torch.equal(got[20000], alone)


def test_a_batch_of_large_matrices_past_two_to_the_31(ac):
    import torch
    b, m, n = 130, 1024, 16384
    assert b * m * n > 1 << 31
    grad = torch.empty((b, m, n), dtype=torch.bfloat16, device="cuda")
    grad[:] = mu.matrix("noise", 1, m, n, 24).bfloat16()
    grad[64] *= -1
    want = mu.plain(grad[:1], None, 0.0, False, 5, 1.0, 1e-7)[1]
    got = mu.run(ac, grad, None, momentum=0.0, nesterov=False)[1]
    for i in (0, 1, 64, 129):
        mu.check(got[i:i + 1] * (-1 if i == 64 else 1), want)


# narrow tiles, lone CTAs, pairs; slices and split tiles over the classes (few tokens) and over the tokens (few classes)
@pytest.mark.parametrize("T,V,D", [(40, 60000, 64), (16, 100003, 72), (3000, 40, 256), (5000, 129, 130), (1000, 4096, 128), (1025, 4096, 64),
                                   (1024, 4097, 64), (33, 1000, 512), (32, 4097, 512), (2048, 5000, 264)])
@pytest.mark.parametrize("mode", ["step", "backward"])
def test_loss_on_both_sides_of_each_choice(ac, T, V, D, mode):
    x = ce.make(T, V, D, True, seed=31)
    want = ce.plain(*x)
    o = ce.run(ac, mode, *x, lse=None if mode == "step" else want["lse"].float())
    if mode == "step":
        ce.check_loss(o, want, D)
    ce.check_grads(o, want, x[3])


def test_weight_gradient_past_two_to_the_31(ac):
    import torch
    T, V, D = 8, 540000, 4096
    assert V * D > 1 << 31
    g = torch.Generator("cuda").manual_seed(32)
    w = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    w[:] = (torch.randn((1, D), generator=g, device="cuda") / 64).bfloat16()
    w[-5000:] = (torch.randn((5000, D), generator=g, device="cuda") / 64).bfloat16()
    h = torch.randn((T, D), generator=g, device="cuda").bfloat16()
    labels = torch.tensor([0, 1, V // 2, V - 1, V - 2, V - 5000, V - 4999, V - 1], device="cuda")
    dloss = torch.full((T,), 0.3, device="cuda")
    x = h.double() @ w[-5000:].double().T
    same = (h.double() @ w[:1].double().T)[:, 0]      # the logit of each of the V - 5000 equal rows
    lse = torch.logsumexp(torch.cat([x, (same + math.log(V - 5000))[:, None]], 1), 1)
    o = ce.run(ac, "step", h, w, None, labels, dloss)
    tol = ce.tol_loss(D, float(x.abs().max()))
    assert float((o["lse"].double() - lse).abs().max()) <= tol
    p = torch.exp(x - lse[:, None]) * 0.3
    rest = torch.exp(same - lse) * 0.3
    hot = torch.zeros((T, 5000), dtype=torch.float64, device="cuda")
    first = torch.zeros((T, 3), dtype=torch.float64, device="cuda")
    for t, y in enumerate(labels.tolist()):
        if y >= V - 5000:
            hot[t, y - (V - 5000)] = 0.3
        else:
            first[t, [0, 1, V // 2].index(y)] = 0.3
    assert float((o["dw"][-5000:].double() - (p - hot).T @ h.double()).norm() / ((p - hot).T @ h.double()).norm()) <= ce.TOL_GRAD
    want = (rest[:, None] - first).T @ h.double()
    got = torch.stack([o["dw"][0], o["dw"][1], o["dw"][V // 2]]).double()
    assert float((got - want).norm() / want.norm()) <= ce.TOL_GRAD
    plain_row = rest @ h.double()
    for r in (2, V // 2 - 1, V - 5001):
        assert float((o["dw"][r].double() - plain_row).norm() / plain_row.norm()) <= ce.TOL_GRAD, r


def test_weights_of_very_different_size(ac):
    """dloss from 1e-30 to 1e30: g is held relative to the largest, in bf16, whose exponents reach as far as fp32's."""
    import torch
    h, w, b, labels, dloss = ce.make(64, 601, 96, True, seed=33, ignored=0)
    dloss = torch.logspace(-6, 6, 64, device="cuda")
    want = ce.plain(h, w, b, labels, dloss)
    o = ce.run(ac, "step", h, w, b, labels, dloss)
    for t in (0, 31, 63):       # each row's gradient by itself: the weight divides out
        assert float((o["dh"][t].double() - want["dh"][t]).norm() / want["dh"][t].norm()) <= ce.TOL_GRAD, t
    ce.check_grads(o, want, labels)
    for s in (1e-30, 1e30):
        one = ce.run(ac, "step", h, w, b, labels, torch.full((64,), s, device="cuda"))
        ref = ce.plain(h, w, b, labels, torch.full((64,), s, device="cuda"))
        ce.check_grads(one, ref, labels)


def test_an_infinite_or_nan_weight_stays_in_its_row(ac):
    import torch
    h, w, b, labels, dloss = ce.make(70, 500, 64, False, seed=34, ignored=0)
    dloss[7], dloss[9] = float("nan"), float("inf")
    o = ce.run(ac, "step", h, w, b, labels, dloss)
    bad = torch.zeros(70, dtype=torch.bool, device="cuda")
    bad[[7, 9]] = True
    assert bool(o["loss"].isfinite().all()) and bool(o["dh"][~bad].isfinite().all())
    assert not bool(o["dh"][7].isfinite().any()) and not bool(o["dh"][9].isfinite().all())


# both sides of the kernel that forms X X^T and its polynomial in one launch: the shorter side, the number of K-tiles, a pair's
# second CTA with few rows or none of the patches full, more matrices than SMs
@pytest.mark.parametrize("b,m,n", [(1, 65, 2560), (1, 65, 2561), (1, 128, 1152), (1, 129, 1000), (2, 130, 1024), (1, 130, 1025), (3, 256, 700),
                                   (1, 257, 700), (1, 1024, 255), (4, 1000, 161), (170, 100, 130), (90, 140, 150), (1, 2560, 128), (2, 300, 97)])
@pytest.mark.parametrize("kind", ["noise", "lowrank"])
def test_update_with_the_square_in_the_same_launch(ac, kind, b, m, n):
    grad = mu.matrix(kind, b, m, n, 41)
    _, want = mu.plain(grad, None, 0.0, False, 5, 1.0, 1e-7)
    _, got = mu.run(ac, grad, None, momentum=0.0, nesterov=False)
    mu.check(got, want)
