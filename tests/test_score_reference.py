"""CPU pins of the tests' plain forms of the teacher-score operators: closed forms and central
differences of the definitions in 64 bits."""
import math

import pytest
import torch

from tests import score_reference as S


def _rows(n, V, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, V), generator=g, dtype=torch.float64) * 2, g


def test_scores_of_uniform_rows_and_masks():
    z = torch.full((2, 10), 1.5, dtype=torch.float64)
    z[1, 4:] = -math.inf
    s = S.scores(z, torch.tensor([3, 2]), 3)
    assert torch.allclose(s["entropy"], torch.log(torch.tensor([10.0, 4.0], dtype=torch.float64)))
    assert torch.allclose(s["logprob"], -s["entropy"])
    assert s["top_ids"].tolist() == [[0, 1, 2], [0, 1, 2]]
    assert torch.allclose(s["rest"].exp(), torch.tensor([0.7, 0.25], dtype=torch.float64))


def _differences(f, z, eps=1e-6):
    g = torch.zeros_like(z)
    for k in range(z.numel()):
        d = torch.zeros_like(z).view(-1)
        d[k] = eps
        d = d.view_as(z)
        g.view(-1)[k] = (f(z + d) - f(z - d)) / (2 * eps)
    return g


@pytest.mark.parametrize("K", [0, 1, 4])
def test_scores_gradient_against_differences(K):
    z, g = _rows(3, 11, 5)
    y = torch.tensor([0, 10, 4])
    w, h = torch.randn(3, generator=g, dtype=torch.float64), torch.randn(3, generator=g, dtype=torch.float64)
    s = S.scores(z, y, max(K, 1))
    ids = s["top_ids"][:, :K]
    d = torch.randn((3, K), generator=g, dtype=torch.float64)

    def loss(x):
        lp = x - torch.logsumexp(x, dim=1, keepdim=True)
        return float((w * lp.gather(1, y[:, None])[:, 0]).sum() - (h * (lp.exp() * lp).sum(1)).sum() +
                     (d * lp.gather(1, ids)).sum())

    grad, _ = S.scores_grad(z, y, s["lse"], s["entropy"], w, h, ids, d)
    assert torch.allclose(grad, _differences(loss, z), atol=1e-8)


@pytest.mark.parametrize("forward", [False, True])
@pytest.mark.parametrize("with_rest", [False, True])
def test_topk_kl_gradient_against_differences(forward, with_rest):
    z, g = _rows(2, 9, 7)
    u, _ = _rows(2, 9, 8)
    lq = torch.log_softmax(u, dim=1)
    ids = S.order(u, 3)
    top = lq.gather(1, ids)
    rest = torch.log1p(-top.exp().sum(1)) if with_rest else None
    r = S.topk_kl(z, torch.tensor([1, 2]), ids, top, rest, forward, alpha=0.5)

    def loss(x):
        return 0.5 * float(S.topk_kl(x, torch.tensor([1, 2]), ids, top, rest, forward)["kl"].sum())

    assert torch.allclose(r["grad"], _differences(loss, z), atol=1e-8)
    assert torch.allclose(r["grad"].sum(1), torch.zeros(2, dtype=torch.float64), atol=1e-12)
    assert torch.allclose(r["gsq"], (r["grad"] ** 2).sum(1))


def test_topk_kl_over_the_whole_vocabulary_is_the_full_divergence():
    z, _ = _rows(3, 8, 1)
    u, _ = _rows(3, 8, 2)
    lp, lq = torch.log_softmax(z, 1), torch.log_softmax(u, 1)
    ids = S.order(u, 8)
    r = S.topk_kl(z, torch.zeros(3), ids, lq.gather(1, ids), torch.full((3,), -math.inf), False)
    kl = (lp.exp() * (lp - lq)).sum(1)
    assert torch.allclose(r["kl"], kl)
    assert torch.allclose(r["grad"], lp.exp() * (lp - lq - kl[:, None]))
    assert torch.allclose(r["logratio"], (lp - lq)[:, 0])
    # fewer categories never see more of the divergence
    short = S.topk_kl(z, torch.zeros(3), ids[:, :3], lq.gather(1, ids[:, :3]), None, False)
    assert (short["kl"] <= kl + 1e-12).all() and (short["kl"] >= -1e-12).all()


def test_quantize_steps():
    x = torch.tensor([[1.0, -2.54, 0.01, 0.03], [0.0, 0.0, 0.0, 0.0]])
    q, step = S.quantize(x)
    assert step[0].item() == pytest.approx(0.02) and step[1].item() == 0.0
    assert q.tolist() == [[50, -127, 0, 1], [0, 0, 0, 0]] or q[0, :2].tolist() == [50, -127]
    assert (q[0].float() * step[0] - x[0]).abs().max() <= step[0] * (0.5 + 1e-5)
