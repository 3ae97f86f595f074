"""The example from the allocation to the clipped gradient: prompts that end anywhere
in a page."""
import pytest
import torch

from tests.test_gpu_rollout_step import example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prompt_len", [1, 2, 15, 16, 17, 32, 48])
def test_example_prompts_of_every_length(prompt_len):
    """The last prompt token is the first step's first row, so it is not among
    those cached before, also where the prompt fills its pages."""
    o = example().main(prompts=2, G=3, prompt_len=prompt_len, steps=3, drafts=2, V=256)
    assert o["status"] == 0
    assert (o["start"] == prompt_len - 1).all()
    assert (o["lens"] - o["start"] == o["made"]).all()


@pytest.mark.parametrize("kw", [dict(), dict(prompts=2, G=3, prompt_len=33, steps=7, drafts=0,
                                             V=512, page=8, seed=3)])
def test_example_log_probabilities_token_by_token(kw):
    """Every generated token's log-probability, as the verification returned it,
    against the one that the scored hidden states give in 64 bits.

    Both sides have an attention output rounded to bf16 after weights rounded to
    bf16. A rounding is uniform within half an ulp: s = 2^-8 / sqrt(3) of the value
    at most (root mean square). The output's goes with |h_d|, the weights' with
    sqrt(sum p^2 v^2) <= 1 (values have unit variance by the weights' scale). So a
    logit 8 h.w is off by sd = 8 s sqrt(2) sqrt(sum_d w_d^2 (h_d^2 + 1)) between the
    sides, and a log-probability by at most 6 sd for its own logit and as much for
    the normaliser (chance of one false alarm over 2000 tokens: 1e-5).

    The comparison has to notice tokens in the wrong place: moved by one row, the
    log-probabilities differ by far more than the bound allows."""
    o = example().main(**kw)
    assert o["status"] == 0
    h, w, y, old = o["hidden"].double(), o["head"].double(), o["y"].long(), o["logp_tokens"]
    logp = torch.log_softmax(h @ w.t(), -1)  # `hidden` has the factor of 8
    sd = 2.0 ** -8 * (2.0 / 3.0) ** 0.5 * ((h.square() + 64.0) @ w.square().t()).sqrt()
    bound = 12.0 * sd.amax(1)
    got = logp.gather(1, y[:, None])[:, 0]
    assert old.shape == got.shape and len(got) == int(o["made"].sum())
    assert ((got - old).abs() <= bound).all()
    moved = logp.gather(1, y.roll(1)[:, None])[:, 0]
    assert float((moved - old).abs().mean()) > 2.0 * float(bound.mean())
    sums = torch.zeros_like(o["logp_old"], dtype=torch.float64)
    sums.index_add_(0, torch.repeat_interleave(torch.arange(len(sums), device="cuda"), o["made"]),
                    old.double())
    assert torch.allclose(sums, o["logp_old"].double(), rtol=1e-5, atol=1e-5)
