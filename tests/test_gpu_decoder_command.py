"""The decoder stack's command: what it prints and refuses."""
import re

import pytest
import torch

from paper_2407_00066_amd import decoder

from _gpu_helpers import say

pytestmark = pytest.mark.gpu


def test_times_with_and_without_the_preparation(capsys):
    say("decoder command")
    decoder.main(["--requests", "2", "--context", "33", "--layers", "1", "--steps", "3"])
    out = capsys.readouterr().out
    for line in ("prompts: 2 x 33 tokens, 1 layers: ", "decode: 2 requests, 1 layers: "):
        found = re.search(re.escape(line) + r"([0-9.]+) ms(?: a step)?, ([0-9.]+) with the batch(?:es)?'s? preparation", out)
        assert found and 0 < float(found[1]) < float(found[2])


@pytest.mark.parametrize("name", ["requests", "context", "layers", "steps"])
def test_counts_of_zero_are_refused(name):
    with pytest.raises(SystemExit):
        decoder.main(["--" + name, "0"])


@pytest.mark.parametrize("counts,kv_len", [([3], [2]), ([1, 5], [9, 4]), ([-1], [4]), ([], [])])
def test_batch_refuses_tokens_before_the_first(counts, kv_len):
    """A sequence's new tokens are among its cached ones: others would be written to pages of later ones."""
    cluster_of = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="counts must be"):
        decoder.Batch([0] * len(counts), cluster_of, 2, 1, counts, kv_len, [[0, 1]] * len(counts), 16)
