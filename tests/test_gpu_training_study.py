"""The training operators run together, as the study uses them (needs an MI355X)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_the_student_learns_and_bsp_is_a_lookahead_of_one():
    from paper_2001_01347_amd import training_study
    bsp = training_study.train(workers=4, supersteps=6, lookahead=1)
    elastic = training_study.train(workers=4, supersteps=6, lookahead=5)
    for rows in (bsp, elastic):
        assert all(math.isfinite(r["loss"]) for r in rows)
        assert rows[-1]["loss"] < rows[0]["loss"]
        assert all(b["barrier"] > a["barrier"] for a, b in zip(rows, rows[1:]))
    assert all(r["iterations"] == 4 for r in bsp)
    assert all(4 <= r["iterations"] <= 20 for r in elastic) and sum(r["iterations"] for r in elastic) > 24


def test_one_worker_is_plain_distillation():
    """A single worker's step against the same step in plain torch operations, in 32 bits: the merge adds its whole push."""
    from paper_2001_01347_amd import training, training_study as ts
    gen = torch.Generator(device="cuda").manual_seed(3)
    teacher, flat = ts.Student.initial(gen), ts.Student.initial(gen)
    x = torch.randn((20, ts.WIDTH), generator=gen, device="cuda")
    index, values, labels = ts._teach(teacher, x)
    leaves = [w.clone().requires_grad_() for w in ts.Student.views(flat)]
    loss = ts._loss(leaves, x, index, values, labels)
    loss.backward()

    plain = [w.double().requires_grad_() for w in ts.Student.views(flat)]
    g, u = x.double() @ plain[0].t(), x.double() @ plain[1].t()
    logits = (torch.nn.functional.silu(g) * u) @ plain[2].t()
    q = torch.softmax(values.double() / ts.TEMPERATURE, dim=1)
    logp = torch.log_softmax(logits / ts.TEMPERATURE, dim=1).gather(1, index)
    nll = -torch.log_softmax(logits, dim=1).gather(1, labels[:, None])[:, 0]
    want = (ts.KL_WEIGHT * ts.TEMPERATURE ** 2 * (q * (q.log() - logp)).sum(dim=1) + ts.CE_WEIGHT * nll).mean()
    want.backward()
    # 32 bits throughout, sums of at most 1000 terms: relative errors of some 1000 steps of 2^-24
    assert abs(loss.item() - want.item()) <= 1000 * 2.0 ** -24 * abs(want.item())
    for a, b in zip(leaves, plain):
        assert (a.grad.double() - b.grad).norm() <= 1000 * 2.0 ** -24 * b.grad.norm()

    push = torch.cat([-0.5 * leaf.grad.reshape(-1) for leaf in leaves])[None]
    out, _, _ = training.ebsp_merge_pushes(flat, push, torch.full((1,), 3, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, flat + push[0])
