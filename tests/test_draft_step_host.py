"""Prompts and trees of the drafting model without a GPU: what it refuses before anything is launched."""
import pytest
import torch

from paper_2604_04701_amd import draft_step as D


@pytest.fixture
def model(monkeypatch):
    """A model of three sequences whose tables hold 40 tokens each, without blocks."""
    monkeypatch.setattr(D, "DEV", "cpu")
    m = object.__new__(D.Model)
    m.S, m.page, m.nodes, m.max_tokens, m.longest, m.vocab = 3, 8, 4, 40, 40, 50
    m.table = torch.arange(15, dtype=torch.int32).view(3, 5)
    m.cos_sin, m.blocks = None, []
    m.adapters, m.lengths = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    m.embedding = torch.zeros(50, 16)
    return m


@pytest.mark.parametrize("starts,tokens", [([0, 41, 42, 43], 43), ([0, 1, 2, 500], 500),          # beyond the table
                                           ([0, 5, 3, 9], 9), ([1, 5, 6, 9], 9), ([0, 5, 9], 9), ([0, 2, 4, 6, 9], 9),       # no starts of three sequences
                                           ([0, 5, 6, 9], 8), ([0, 0, 0, 0], 0)])          # other tokens than starts say
def test_prompts_that_are_refused(model, starts, tokens):
    with pytest.raises(ValueError):
        model.prompt(torch.zeros(tokens, dtype=torch.int32), starts)
    assert model.lengths.tolist() == [0, 0, 0]


def test_a_prompt_may_fill_its_table(model, monkeypatch):
    seen = []
    monkeypatch.setattr(D, "run_step", lambda stack, rows, x: (seen.append(rows), x, [])[1:])
    model.prompt(torch.zeros(57, dtype=torch.int32), [0, 40, 40, 57])
    assert seen[0].slots[:57].tolist() == [*range(40), *range(80, 97)] and model.lengths.tolist() == [40, 0, 17] and model.longest == 40


@pytest.mark.parametrize("window", [1, 256, 360])
def test_a_window_that_the_trees_would_not_have_is_refused(monkeypatch, capsys, window):
    """The nodes of a tree see all tokens: prompts within a window and trees without one are two models."""
    # 300 tokens, 9 rounds of trees of 16 nodes that are 5 deep, and a tree: 361
    monkeypatch.setattr("sys.argv", ["draft_step", "--prompt", "300", "--nodes", "16", "--branch", "2", "--rounds", "8", "--window", str(window)])
    monkeypatch.setattr(D.B, "muxq_init", lambda: pytest.fail("not refused"))
    with pytest.raises(SystemExit):
        D.main()
    assert "window" in capsys.readouterr().err


def test_trees_behind_a_windowed_prompt_warn(model, monkeypatch):
    monkeypatch.setattr(D, "run_step", lambda stack, rows, x: (x, []))
    model.at_round, model.depths = D.Rows(model, None), torch.arange(4)
    model.longest = 20
    model.prompt(torch.zeros(30, dtype=torch.int32), [0, 20, 25, 30], window=24)
    model.place()                                     # nothing is beyond 24 tokens
    model.prompt(torch.zeros(30, dtype=torch.int32), [0, 20, 25, 30], window=23)
    with pytest.warns(UserWarning, match="window of 23"):
        model.place()
