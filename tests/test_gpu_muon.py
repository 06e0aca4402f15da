"""The orthogonalised update (ac_muon_update) against a plain 64-bit implementation.

Tolerances. v' is one fp32 multiply-add: 2^-23 of the larger term. The update is rounded to bf16 once (2^-9 of each entry
at most); before that, the products' operands are rounded to fp16 (2^-12). A rounding of A or P of that size changes X by
2^-12 |A| |X| in directions that the steps neither shrink nor (X itself being carried with 22 bits) amplify beyond a = 3.4445
each, and five steps of two such roundings add to about sqrt(10) 2^-12 * 2 = 1.6e-3 of the result's norm."""
import math

import pytest

import __graft_entry__ as entry

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -9 + 1.6e-3
ABC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def ac():
    entry.build()
    import paper_2409_11902_b200 as ac
    return ac


def matrix(kind, b, m, n, seed):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    if kind == "noise":
        return randn(b, m, n)
    if kind == "lowrank":
        r = max(1, min(m, n) // 8)
        return randn(b, m, r) @ randn(b, r, n) + 0.05 * randn(b, m, n)
    k = min(m, n)       # singular values from 1 to 1e-3
    q, p = torch.linalg.qr(randn(b, m, k))[0], torch.linalg.qr(randn(b, n, k))[0]
    return (q * torch.logspace(0, -3, k, device="cuda")) @ p.mT


def plain(grad, v, beta, nesterov, steps, scale, eps, abc=ABC):
    g = grad.double()
    v = None if v is None else beta * v.double() + g
    u = g if v is None else g + beta * v if nesterov else v
    x = u / (u.square().sum((1, 2), keepdim=True).sqrt() + eps)
    a, b, c = abc
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * s @ s) @ x
    return v, scale * x


def run(ac, grad, v, out=None, stream=None, **kw):
    import torch
    b, m, n = grad.shape
    d = ac.MuonDesc(m, n, batch=b, dtype="bf16" if grad.dtype == torch.bfloat16 else "f32", **kw)
    ws = torch.full((ac.ac_muon_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    update = torch.full((b, m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(v, float("nan")) if v is not None and out is None else out
    ac.ac_muon_update(d, grad, v, out, update, ws, stream=stream)
    assert ac.ac_workspace_status(ws, stream) == (0, 0)
    return out, update


def check(got, want, tol=TOL):
    for i in range(len(got)):       # each matrix by itself
        err = float((got[i].double() - want[i]).norm() / want[i].norm())
        assert err <= tol, (i, err)


SIZES = [(1, 1, 1), (1, 1, 9), (1, 9, 1), (2, 8, 8), (3, 16, 40), (1, 40, 16), (2, 33, 17), (1, 64, 576), (1, 64, 147), (5, 127, 130),
         (1, 128, 128), (2, 129, 257), (6, 256, 2304), (2, 1024, 256), (1, 2304, 256), (1, 771, 1543), (1, 1543, 515), (1, 640, 5000),
         (2, 3000, 640), (1, 1100, 2300), (1, 2600, 2500)]


@pytest.mark.parametrize("b,m,n", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_update_matches_the_definition(ac, b, m, n, dtype):
    grad, v = matrix("noise", b, m, n, 1), 3 * matrix("noise", b, m, n, 2)
    if dtype == "bf16":
        grad = grad.bfloat16()
    scale = math.sqrt(max(1.0, m / n))
    want_v, want = plain(grad, v, 0.95, True, 5, scale, 1e-7)
    got_v, got = run(ac, grad, v, momentum=0.95, scale=scale)
    assert float((got_v.double() - want_v).abs().max()) <= 2.0 ** -23 * float(want_v.abs().max()) * 2
    check(got, want)


@pytest.mark.parametrize("kind", ["lowrank", "spread"])
@pytest.mark.parametrize("b,m,n", [(1, 64, 576), (2, 256, 1024), (1, 1024, 256), (1, 520, 520), (1, 96, 4608), (1, 1500, 2200)])
def test_uneven_spectra(ac, kind, b, m, n):
    grad = matrix(kind, b, m, n, 7)
    _, want = plain(grad, None, 0.0, False, 5, 1.0, 1e-7)
    _, got = run(ac, grad, None, momentum=0.0, nesterov=False)
    check(got, want)


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 6, 8])
@pytest.mark.parametrize("nesterov", [False, True])
def test_steps_and_momentum_forms(ac, steps, nesterov):
    grad, v = matrix("noise", 2, 72, 200, 3), matrix("noise", 2, 72, 200, 4)
    want_v, want = plain(grad, v, 0.9, nesterov, steps, 0.2, 1e-7)
    got_v, got = run(ac, grad, v.clone(), momentum=0.9, nesterov=nesterov, steps=steps, scale=0.2)
    assert float((got_v.double() - want_v).abs().max()) <= 2.0 ** -22 * float(want_v.abs().max())
    check(got, want)


def test_other_coefficients(ac):
    grad = matrix("noise", 1, 100, 300, 5)
    abc = (15 / 8, -10 / 8, 3 / 8)
    _, want = plain(grad, None, 0.0, False, 7, 1.0, 1e-7, abc)
    _, got = run(ac, grad, None, momentum=0.0, steps=7, coefficients=abc)
    check(got, want)


def test_momentum_in_place_equals_out_of_place(ac):
    import torch
    grad, v = matrix("noise", 3, 50, 70, 6), matrix("noise", 3, 50, 70, 7)
    a_v, a = run(ac, grad, v)
    w = v.clone()
    b_v, b = run(ac, grad, w, out=w)
    assert torch.equal(a_v, b_v) and torch.equal(a, b)


def test_scales_of_the_gradient_do_not_matter(ac):
    grad = matrix("noise", 1, 80, 240, 8)
    _, want = plain(grad, None, 0.0, False, 5, 1.0, 0.0)
    for s in (2.0 ** -40, 2.0 ** 40):
        _, got = run(ac, grad * s, None, momentum=0.0, eps=0.0)
        check(got, want)


def test_zero_gradient_and_bad_matrices_stay_by_themselves(ac):
    import torch
    grad = matrix("noise", 4, 60, 90, 9)
    clean = run(ac, grad, None, momentum=0.0)[1]
    grad[1] = 0
    grad[2, 5, 5] = float("nan")
    _, got = run(ac, grad, None, momentum=0.0)
    assert bool((got[1] == 0).all()) and bool(got[2].isnan().any())
    assert torch.equal(got[0], clean[0]) and torch.equal(got[3], clean[3])


@pytest.mark.parametrize("b,m,n", [(1, 64, 576), (2, 300, 700), (1, 2600, 2500)])
def test_deterministic_on_another_stream(ac, b, m, n):
    import torch
    grad, v = matrix("noise", b, m, n, 10), matrix("noise", b, m, n, 11)
    first = run(ac, grad, v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = run(ac, grad, v, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
