"""The command that runs prompts and rounds of drafted trees."""
import re

import pytest

from block_common import say
from paper_2604_04701_amd import draft_step as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("more", [[], ["--fp16-cache", "--window", "1000"]])
def test_the_command_runs(monkeypatch, capsys, more):
    say(f"[draft] command {more}")
    monkeypatch.setattr("sys.argv", ["draft_step", "--width", "256", "--heads", "4", "--blocks", "2", "--batch", "3", "--prompt", "50", "--nodes", "7",
                                     "--rounds", "2", "--vocab", "501", *more])
    D.main()
    said = capsys.readouterr().out
    us, kept = re.search(r"(\d+) us a round, ([\d.]+) tokens", said).groups()
    assert int(us) > 0 and 1.0 <= float(kept) <= 3.0              # (the last token always stands; trees are three deep)
