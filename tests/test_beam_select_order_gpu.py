"""Beam search's selection (rwkvq_beam_select): the order of the candidates, place by place."""
import math

import pytest
import torch

from tests import test_beam_gpu as S

pytestmark = pytest.mark.gpu

LOWEST = torch.finfo(torch.float32).min


def same_places(logits, scores, picks):
    """Parents, tokens and scores are those of the definition, all of them."""
    V = logits.shape[1]
    ns, pa, to, _ = S.select(logits, scores, picks, eos=V - 1)
    ref = S.totals(logits, scores, None, V - 1)
    best, at = S.order(ref, logits, V)
    assert torch.equal(pa.long() * V + to.long(), at[:, :picks]), (pa.tolist(), to.tolist(), at[:, :picks].tolist())
    return ns, best[:, :picks]


@pytest.mark.parametrize("best", [0, 3, 7])
@pytest.mark.parametrize("K,V,kept,picks", [(8, 20000, 1, 16), (8, 20000, 0, 16), (8, 300, 1, 16), (8, 70000, 3, 64), (64, 3000, 1, 64)])
def test_totals_below_fp32(K, V, kept, picks, best):
    """Masks of the type's lowest value under low scores: the totals have no fp32 number, which says nothing about their order."""
    g = torch.Generator().manual_seed(K + V + best)
    logits = torch.full((2 * K, V), LOWEST)
    for row in logits:
        row[torch.randperm(V, generator=g)[:kept]] = torch.randn(kept, generator=g)
    if kept == 0:
        logits[:, V // 2] = 0.0
    # scores a thirty-second apart from one another, relative to them: far more than anything beside the mask
    scores = -1e38 * (1.0 + torch.stack([torch.randperm(K, generator=g) for _ in range(2)]).float() / 32)
    at = scores.argmax(1)
    for r in range(2):          # the best beam's candidates stand among the first, in the middle, or behind all others
        scores[r, best], scores[r, at[r]] = scores[r, at[r]].clone(), scores[r, best].clone()
    ns, want = same_places(logits, scores, picks)
    # as many as are not masked have totals that fp32 has numbers for
    assert torch.equal(ns, want.float()) and torch.isinf(ns).sum().item() == 2 * max(0, picks - K * max(kept, 1))


@pytest.mark.parametrize("dtype", S.TYPES)
@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_ties_within_beams_that_lie_apart(dtype, V):
    """Logits of three values, beams a hundredth apart or more: equal ones by their tokens, the beams by their totals."""
    g = torch.Generator().manual_seed(V)
    row = torch.randint(0, 3, (V,), generator=g).float()
    # the same values in another order, so that the sums are the same to a few roundings and the scores alone tell the beams apart
    logits = torch.stack([row[torch.randperm(V, generator=g)] for _ in range(6)]).to(S.TYPES[dtype])
    for scores in (torch.tensor([[0.0, -0.01, -2.0], [-3.0, -2.99, -3.01]]), torch.tensor([[-1.0, -2.0, -3.0], [-9.0, -8.0, -1.0]])):
        ns, want = same_places(logits, scores, 12)
        assert ((ns.double() - want).abs() <= S.LSE + 2.0 ** -23 * want.abs()).all()


@pytest.mark.parametrize("dtype", S.TYPES)
@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_ties_of_beams_that_are_the_same(dtype, V):
    """The same logits and scores: by beam, then by token, from the first place to the last."""
    g = torch.Generator().manual_seed(V)
    row = torch.randint(0, 3, (V,), generator=g).to(S.TYPES[dtype])
    top = torch.nonzero(row == row.max()).flatten()
    picks = 24
    ns, pa, to, _ = S.select(row.repeat(3, 1), torch.full((1, 3), -1.5), picks, eos=0)
    level = [(k, int(v)) for k in range(3) for v in top]
    rest = [(k, int(v)) for k in range(3) for v in torch.nonzero(row == row.max() - 1).flatten()]
    assert list(zip(pa[0].tolist(), to[0].tolist())) == (level + rest)[:picks]
    assert (ns[0].double() - S.totals(row.view(1, -1), torch.tensor([[-1.5]]), None, 0)[0, to[0].long()]).abs().max() <= S.LSE + 2.0 ** -20
    assert not math.isinf(float(ns.min()))
