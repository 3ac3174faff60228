"""The decoder stack's command: what it prints and refuses."""
import re

import pytest

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
