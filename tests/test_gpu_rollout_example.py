"""The example from the allocation to the clipped gradient: prompts that end anywhere
in a page."""
import pytest

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
