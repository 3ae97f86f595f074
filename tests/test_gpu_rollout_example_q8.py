"""The example with its cache in 8 bits: from the allocation to the clipped gradient."""
import pytest
import torch

from tests.test_gpu_rollout_step import example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.int8, torch.float8_e4m3fn])
def test_example_over_a_cache_in_8_bits(dtype):
    """Every generated token's log-probability, as the verification returned it, against
    the one that the hidden states of whole rollouts give in 64 bits: both attend over
    the same stored values, so the bound is that of the example over a bf16 cache. A
    rounding to bf16 is uniform within half an ulp, s = 2^-8 / sqrt(3) of the value at
    most (root mean square); each side has one of its output and one of each weight, the
    latter with sqrt(sum p^2 v^2) <= 1 (a stored value is off by 2^-4 of itself at most:
    1.07). A logit 8 h.w is off by sd = 8 s sqrt(2) sqrt(sum_d w_d^2 (h_d^2 + 1.07^2))
    between the sides, a log-probability by 6 sd for its own logit and as much for the
    normaliser. And the gradient is the one of the surrogate at these hidden states."""
    o = example().main(prompts=2, G=4, prompt_len=37, steps=6, drafts=2, V=512,
                       cache_dtype=dtype)
    assert o["status"] == 0
    assert (o["lens"] - o["start"] == o["made"]).all() and int(o["made"].sum()) > 0
    h, w, y, old = o["hidden"].double(), o["head"].double(), o["y"].long(), o["logp_tokens"]
    logp = torch.log_softmax(h @ w.t(), -1)
    sd = 2.0 ** -8 * (2.0 / 3.0) ** 0.5 * ((h.square() + 64.0 * 1.15) @ w.square().t()).sqrt()
    got = logp.gather(1, y[:, None])[:, 0]
    assert ((got - old).abs() <= 12.0 * sd.amax(1)).all()
    # d/dh of sum_i c_i log pi(o_i): c (w_y - sum_v p_v w_v) in each row.
    rows = torch.repeat_interleave(torch.arange(len(o["coef"]), device="cuda"), o["made"])
    c = o["coef"].double()[rows]
    want = c[:, None] * (w[y] - logp.exp() @ w)
    assert float((o["dH"].double() - want).norm()) <= 4e-3 * max(float(want.norm()), 1e-30)
