"""The training step with the library's own classifier loss and weight update (train_step's head="fused",
optimizer="muon"): the same loss and gradients as the framework's head up to bf16 rounding, updates that are what the
formula says of the gradients the step really produced, and a loss that falls."""
import pytest

import __graft_entry__ as entry

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def test_fused_head_matches_the_framework_head():
    import torch
    import torch.nn.functional as F
    from paper_2409_11902_b200.train_step import LinearCrossEntropy
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn((64, 2048), generator=g, device="cuda", requires_grad=True)
    w = (torch.randn((1000, 2048), generator=g, device="cuda") / 45).requires_grad_(True)
    b = torch.randn(1000, generator=g, device="cuda", requires_grad=True)
    labels = torch.randint(0, 1000, (64,), generator=g, device="cuda")
    labels[::7] = -100
    loss = LinearCrossEntropy.apply(x, w, b, labels)
    (3 * loss).backward()
    got = [t.grad.double() for t in (x, w, b)]
    # the same function of the bf16 operands in 64 bits
    ref = [t.detach().bfloat16().double().requires_grad_(True) for t in (x, w, b)]
    want = F.cross_entropy(F.linear(*ref), labels, ignore_index=-100)
    (3 * want).backward()
    assert abs(float(loss) - float(want)) <= 1e-5 * float(want)
    for a, r in zip(got, ref):
        # g rounded to bf16, the result, and (x's gradient) its product with the upstream 3: three roundings of 2^-9
        assert float((a - r.grad).norm() / r.grad.norm()) <= 3 * 2.0 ** -9


def test_step_with_both_operators_agrees_with_the_framework_step():
    from paper_2409_11902_b200 import train_step
    runs = {h: train_step.training_step("compressed+mask", batch=8, k=2, device="cuda:0", head=h) for h in ("framework", "fused")}
    # the framework rounds its logits to bf16 (2^-9 of logits of order one), the fused head does not
    assert runs["fused"]["loss"] == pytest.approx(runs["framework"]["loss"], abs=2.0 ** -6)
    assert runs["fused"]["grad_norm"] == pytest.approx(runs["framework"]["grad_norm"], rel=0.05)


def test_updates_are_the_orthogonalised_gradients_and_the_loss_falls():
    import torch
    from paper_2409_11902_b200 import train_step
    dev = torch.device("cuda:0")
    model = train_step.ResNet50("compressed+mask", 2, dev, seed=0)
    opt = train_step.Muon(model.params, lr=0.02, sgd_lr=0.02)
    assert sum(len(g["params"]) for g in opt.groups) == 53
    images, labels = train_step.synthetic_batch(16, dev)
    losses = []
    for i in range(6):
        opt.zero_grad()
        loss = model.loss(images, labels, "fused")
        loss.backward()
        losses.append(float(loss.detach()))
        if i == 0:
            before = {id(p): p.detach().clone() for g in opt.groups for p in g["params"]}
            grads = {id(p): p.grad.detach().clone() for g in opt.groups for p in g["params"]}
        opt.step()
        if i > 0:
            continue
        for g in opt.groups:
            for p in g["params"][:1]:
                u = grads[id(p)].double().permute(0, 2, 3, 1).reshape(p.shape[0], -1)
                x = u / (u.norm() + 1e-7)       # the first step: u = (1 + momentum) g, its scale does not matter
                for _ in range(5):
                    s = x @ x.mT
                    x = 3.4445 * x + (-4.7750 * s + 2.0315 * s @ s) @ x
                x = x * max(1.0, p.shape[0] / u.shape[1]) ** 0.5 * -0.02
                step = (p.detach() - before[id(p)]).double().permute(0, 2, 3, 1).reshape(u.shape)
                # bf16 update (2^-9), fp16 products (1.6e-3), and the fp32 subtraction from a weight some hundred times larger
                assert float((step - x).norm() / x.norm()) <= 2.0 ** -9 + 1.6e-3 + 1e-4, tuple(p.shape)
    assert all(l == l for l in losses) and losses[-1] < 0.8 * losses[0], losses
