"""What PromptDecoder.set_chunk takes: refused before a buffer changes where sizes do not fit,
and starts as the kernels take them (inside the tokens, ascending), so that lengths count
what is appended.  Host tensors: no GPU is needed."""
import pytest
import torch

from test_abi import L  # noqa: F401  (the library's binding)


@pytest.fixture(params=["all", "last"])
def dec(L, request):
    from paper_2609_20734_amd import decoder as PD
    shape = PD.DecoderShape(1, 64, 2, 1, 64, 64, 96)
    k = torch.zeros(1, 12, 1, 8, 16, 8, dtype=torch.bfloat16)
    seq = torch.tensor([7, 0, 30], dtype=torch.int32)
    d = PD.PromptDecoder(shape, {}, 3, 10, k, torch.zeros_like(k), torch.zeros(3, 4, dtype=torch.int32), seq, 4, 64, 12,
                         score=request.param)
    d.set_chunk(i32([5, 6]), i32([0, 1, 1, 2]), i32([6, 7]))         # one row each of the first and last request
    return d


def i32(x):
    return torch.tensor(x, dtype=torch.int32)


def test_a_chunk(dec):
    assert dec.seq_lens.tolist() == [8, 0, 31] and dec.row_start.tolist() == [0, 1, 1, 2]
    assert dec.tokens.tolist() == [5, 6] + [0] * 8 and dec.targets.tolist() == [6, 7] + [-1] * 8


@pytest.mark.parametrize("starts,taken", [
    ([0, 6, 2, 8], [0, 6, 6, 8]),               # descending: the request between has no rows
    ([3, 1, 0, 2], [3, 3, 3, 3]),
    ([-5, 2, 4, 8], [0, 2, 4, 8]),
    ([0, 2, 4, 9], [0, 2, 4, 8]),               # beyond the tokens, inside the buffers
    ([0, 2, 2 ** 31 - 1, 8], [0, 2, 8, 8]),
    ([2, 4, 4, 7], [2, 4, 4, 7]),               # tokens in front and behind are no request's
    ([0, 0, 0, 0], [0, 0, 0, 0])])
def test_starts_are_taken_as_the_kernels_take_them(dec, starts, taken):
    was = dec.seq_lens.clone()
    dec.set_chunk(torch.arange(1, 9), i32(starts))
    assert dec.row_start.tolist() == taken
    count = [b - a for a, b in zip(taken, taken[1:])]
    assert (dec.seq_lens - was).tolist() == count
    if dec.listed is not None:
        with_rows = [b for b in range(3) if count[b] > 0]
        assert int(dec.n_listed) == len(with_rows)
        assert dec.listed[:len(with_rows)].tolist() == [taken[b + 1] - 1 for b in with_rows]


def test_a_chunk_of_no_tokens(dec):
    was = dec.seq_lens.tolist()
    dec.set_chunk(i32([]), i32([0, 0, 4, 4]))
    assert dec.seq_lens.tolist() == was and dec.row_start.tolist() == [0] * 4


@pytest.mark.parametrize("n,starts,targets", [
    (11, [0, 4, 8, 11], None),
    (4, [0, 2, 4], None), (4, [0, 1, 2, 3, 4], None), (4, [], None),
    (4, [0, 1, 2, 4], 1), (4, [0, 1, 2, 4], 3), (4, [0, 1, 2, 4], 5), (4, [0, 1, 2, 4], 0)])
def test_refused_before_anything_changes(dec, n, starts, targets):
    names = ("seq_lens", "row_start", "tokens", "targets", "listed", "n_listed")
    was = {k: getattr(dec, k).clone() for k in names if getattr(dec, k) is not None}
    with pytest.raises(ValueError):
        dec.set_chunk(torch.ones(n, dtype=torch.int32), i32(starts), None if targets is None else torch.ones(targets, dtype=torch.int32))
    for k, x in was.items():
        assert torch.equal(getattr(dec, k), x), k
