"""The batch of the decode step without a GPU: positions, slots, and where it ends."""
import pytest
import torch

from paper_2604_04701_amd import decode_block as D


def make(monkeypatch, lengths, most, page=16):
    monkeypatch.setattr(D, "DEV", "cpu")
    g = torch.Generator()
    g.manual_seed(1)
    return D.Batch(g, len(lengths), lengths, most, page, 64, 2, True)


def test_tokens_go_to_the_places_of_the_table(monkeypatch):
    batch = make(monkeypatch, [0, 15, 30], 35)
    for step in range(4):
        at = [n + step for n in (0, 15, 30)]
        assert batch.positions.tolist() == at and batch.lengths.tolist() == [n + 1 for n in at]
        assert batch.slots.tolist() == [int(batch.table[s, n // 16]) * 16 + n % 16 for s, n in enumerate(at)]
        batch.next_token()


@pytest.mark.parametrize("most", [32, 35, 48])
def test_no_token_beyond_the_bound(monkeypatch, most):
    # a position beyond it has no angle, no weight in the attention and, a page later, no entry in the table
    batch = make(monkeypatch, [3, 30], most)
    for _ in range(most - 31):
        batch.next_token()
    assert batch.lengths.max() == most
    before = batch.positions.clone()
    with pytest.raises(ValueError, match=str(most)):
        batch.next_token()
    assert torch.equal(batch.positions, before)


def test_no_sequence_beyond_the_bound(monkeypatch):
    with pytest.raises(ValueError, match="32"):
        make(monkeypatch, [3, 32], 32)
