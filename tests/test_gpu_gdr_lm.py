"""The small gated-delta language model: training lowers its loss, and what beam search returns is
what the whole-sequence forward says of it.

Tolerance of the scores: a float32 mixer's outputs differ by some 1e-6 relative between the forms over
chunks and token by token, logits of size up to about 20 by 1e-4 at the very most, and 12 tokens' log-
probabilities add: 2e-3."""

import pytest
import torch

from paper_2609_07816_amd import gdr_lm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def trained():
    torch.manual_seed(1)
    model = gdr_lm.GdrLM().cuda()
    return model, gdr_lm.train(model, 150, torch.Generator().manual_seed(1))


def test_training_lowers_the_loss(trained):
    losses = trained[1]
    assert torch.isfinite(losses).all()
    assert losses[0] > 3.0  # near log(64) = 4.16 before training
    assert losses[-10:].mean() < 0.25 * losses[0]


@pytest.mark.parametrize("beams,end_token", [(1, 0), (4, 0), (5, 7)])
def test_scores_are_those_of_the_whole_sequence(trained, beams, end_token):
    model = trained[0]
    full = gdr_lm.repeated(3, 80, 20, 64, torch.Generator().manual_seed(beams))
    prompts = [full[0][:25], full[1][:1], full[2][:70]]
    steps = 12
    tokens, scores = model.beam_search(prompts, steps, beams, end_token)
    assert (scores.diff(dim=1) <= 0).all()
    for n, p in enumerate(prompts):
        seqs = torch.cat([p.cuda().expand(beams, -1), tokens[n]], 1)
        assert torch.unique(seqs, dim=0).shape[0] == beams
        with torch.no_grad():
            logp = torch.log_softmax(model(seqs[:, :-1]), -1)[:, p.numel() - 1:]
        each = logp.gather(-1, tokens[n].long()[..., None])[..., 0]
        ended = (tokens[n] == end_token).int().cumsum(1) - (tokens[n] == end_token).int() > 0
        want = each.masked_fill(ended, 0.0).sum(-1)
        assert torch.allclose(scores[n], want, atol=2e-3, rtol=0)


def test_the_best_beam_continues_the_string(trained):
    full = gdr_lm.repeated(4, 80, 20, 64, torch.Generator().manual_seed(3))
    tokens, _ = trained[0].beam_search([x[:45] for x in full], 15, 4)
    assert (tokens[:, 0].cpu() == full[:, 45:60]).float().mean() > 0.8
