"""GPU: new tokens placed in a paged cache: tables, stacks, lengths, starts, owners and slots equal to a program's that goes through the sequences one by one."""
import random

import pytest
import torch

import serving_plain as P
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _state(rng, n, page, most, spare, width=None):
    lengths = [rng.choice((0, page, rng.randint(0, most))) for _ in range(n)]
    width = width or -(-most // page) + 3
    counts = [-(-length // page) for length in lengths]
    deal = rng.sample(range(sum(counts) + spare), sum(counts) + spare)
    pages, at = [[-7] * width for _ in range(n)], 0
    for row, c in zip(pages, counts):
        row[:c] = deal[at:at + c]
        at += c
    return pages, lengths, deal[at:] + [-9] * at, spare


def _check(pages, page, lengths, new, free, n_free, n_tokens, ends=None, in_place=False):
    want = P.place(pages, page, lengths, new, free, n_free, n_tokens, ends)
    table, held, stack, count, status = torch.tensor(pages, dtype=torch.int32, device=DEV).view(len(pages), -1), ints(lengths), ints(free), ints([n_free]), ints([0, 0])
    kept = dict(lengths_out=held, n_free_out=count) if in_place else {}
    got = B.place_tokens(table, page, held, ints(new), stack, count, n_tokens, ends=None if ends is None else ints(ends), status=status, **kept)
    slots, starts, after, owners, left, want_table, want_stack, told = want
    assert got.slots.dtype == torch.int64 and got.slots.tolist() == slots
    assert got.starts.tolist() == starts and got.lengths.tolist() == after and got.owners.tolist() == owners and got.n_free.tolist() == [left]
    assert table.tolist() == want_table and stack.tolist() == want_stack
    assert status.tolist() == ([1, told] if told else [0, 0])
    assert (got.lengths is held) == in_place and (in_place or (held.tolist() == list(lengths) and count.tolist() == [n_free]))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,page,most,new", [(1, 16, 40, 1), (1, 64, 3000, 2999), (16, 64, 4000, 1), (63, 16, 200, 300), (64, 32, 100, 5), (65, 256, 1000, 700), (300, 16, 50, 90),
                                             (1023, 16, 20, 1), (1025, 16, 40, 20), (3000, 16, 33, 3)])
def test_any_step(n, page, most, new, in_place):
    for seed in range(4):
        rng = random.Random(seed * 1000 + n)
        fresh = [rng.choice((0, 1, rng.randint(0, new))) for _ in range(n)]
        ends = None if seed == 0 else [int(rng.random() < 0.3) * rng.choice((1, -5)) for _ in range(n)]
        # enough pages, a few, none
        spare = (sum(fresh) // page + 2 * n, sum(fresh) // page + 2 * n, rng.randint(0, 9), 0)[seed]
        pages, lengths, free, n_free = _state(rng, n, page, most, spare, -(-(most + new) // page) + 1)
        _check(pages, page, lengths, fresh, free, n_free, sum(fresh) + rng.choice((0, 1, 77)), ends, in_place)


def test_a_sequence_begins_anew_in_pages_that_it_gave_back():
    _check([[3, 5, 1]], 16, [40], [33], [-1] * 3, 0, 33, [1])
    _check([[3, 5, 1], [0, 2, 4]], 16, [40, 16], [48, 5], [-1] * 4, 0, 60, [1, 0])


@pytest.mark.parametrize("new,n_tokens", [([5, -1, 3], 9), ([5, 100, 3], 200), ([5, 4, 3], 11), ([5, 4, 3], 4), ([0, 0, 0], 0), ([2**31 - 1, 2**31 - 1, 1], 5)])
def test_sequences_that_get_nothing(new, n_tokens):
    """Fewer than none, more than a row of the table has room for, more than there are slots: the others get theirs."""
    _check([[0, 1, -7], [2, -7, -7], [-7, -7, -7]], 16, [20, 16, 0], new, [3, 4, 5, 6, 7, -9], 5, n_tokens)


def test_pages_run_out():
    """A sequence that needs none of them goes on behind one that got none."""
    _check([[0, -7], [1, -7], [2, -7], [3, -7]], 16, [16, 3, 16, 16], [1, 13, 1, 1], [9, 8, -1, -1], 1, 20)


def test_no_sequences_and_no_tokens():
    got = B.place_tokens(torch.empty(0, 4, dtype=torch.int32, device=DEV), 16, ints([]), ints([]), ints([1, 2]), ints([2]), 3)
    assert got.slots.tolist() == [-1] * 3 and got.starts.tolist() == [0] and got.owners.tolist() == [-1] * 3 and got.n_free.tolist() == [2]
    got = B.place_tokens(ints([[1]]), 16, ints([4]), ints([0]), ints([]), ints([0]), 0)
    assert got.slots.shape == (0,) and got.starts.tolist() == [0, 0] and got.lengths.tolist() == [4]


def test_numbers_out_of_range_are_told():
    """Lengths that no table has, a stack that is larger than its room or overflows, pages below 0: nothing outside is touched."""
    status = ints([0, 0])
    table, stack = ints([[4, 5], [6, 7], [-3, -3]]), ints([1, 2, 3])
    got = B.place_tokens(table, 16, ints([33, -1, 5]), ints([1, 1, 2]), stack, ints([77]), 8, status=status)
    assert got.slots.tolist() == [-1] * 8 and got.lengths.tolist() == [33, -1, 7] and got.n_free.tolist() == [3] and got.owners.tolist() == [0, 1, 2, 2] + [-1] * 4
    assert status.tolist() == [1, 5] and table.tolist() == [[4, 5], [6, 7], [-3, -3]] and stack.tolist() == [1, 2, 3]
    status.zero_()
    got = B.place_tokens(table, 16, ints([2**31 - 1, -5, 5]), ints([0, 17, 0]), stack, ints([2]), 20, ends=ints([1, 1, 0]), status=status)
    # (of the first one's pages one finds room, the second gives none back)
    assert stack.tolist() == [1, 2, 4] and status.tolist() == [1, 3] and got.lengths.tolist() == [0, 17, 5] and got.n_free.tolist() == [1]
    assert table.tolist() == [[4, 5], [4, 2], [-3, -3]] and got.slots.tolist() == [4 * 16 + i for i in range(16)] + [2 * 16] + [-1] * 3


def test_on_another_stream():
    rng = random.Random(5)
    pages, lengths, free, n_free = _state(rng, 40, 16, 100, 90)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _check(pages, 16, lengths, [7] * 40, free, n_free, 280)
    side.synchronize()


@pytest.mark.parametrize("n", [5, 60, 400])
def test_a_call_made_again_gives_the_same(n):
    """With outputs of their own, where no sequence that ends gets tokens (a refused one gets none); in one workgroup and in three launches."""
    rng = random.Random(n)
    pages, lengths, free, n_free = _state(rng, n, 16, 90, n)
    ends = [int(s % 4 == 1) for s in range(n)]
    new = [0 if e else rng.randint(0, 30) for e in ends]
    ends[-1], new[-1] = 1, 10 ** 6
    table, held, stack, count, status = torch.tensor(pages, dtype=torch.int32, device=DEV), ints(lengths), ints(free), ints([n_free]), ints([0, 0])
    call = lambda: [t.clone() for t in (*B.place_tokens(table, 16, held, ints(new), stack, count, 40 * n, ends=ints(ends), status=status), table, stack)]  # noqa: E731
    first = call()
    assert first[2].tolist()[-1] == 0 and int(status[1]) >= 1 and (first[0] >= 0).any()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(call(), first))


def test_a_sequence_that_ends_and_gets_tokens_has_its_new_pages_at_once():
    """Its row begins with what it was dealt, so what it gave back is in the stack alone, and the same call on this table would be another one."""
    table, stack = ints([[3, 5, 1]]), ints([-1, -1, -1])
    got = B.place_tokens(table, 16, ints([40]), ints([20]), stack, ints([0]), 20, ends=ints([1]))
    assert table.tolist() == [[1, 5, 1]] and stack.tolist() == [3, 5, 1] and got.n_free.tolist() == [1] and got.slots.tolist() == [*range(16, 32), *range(80, 84)]


@pytest.mark.parametrize("n", [1, 7, 60, 300, 1500])
def test_the_last_tokens_of_sequences(n):
    """Where each sequence's last new token is; -1 for those without one and for those that get nothing.  Nothing else is changed by asking for it."""
    for seed in range(3):
        rng = random.Random(seed * 100 + n)
        pages, lengths, free, n_free = _state(rng, n, 16, 60, (2 * n, n // 3, 0)[seed], 9)
        new = [rng.choice((0, 1, 25, -1, 10 ** 6 if rng.random() < 0.05 else 3)) for _ in range(n)]
        ends = None if seed == 0 else [int(rng.random() < 0.3) for _ in range(n)]
        n_tokens = sum(v for v in new if v < 10 ** 6 and v > 0) * (4 if seed else 1)
        results = []
        for last in (None, ints([77] * n)):
            table, stack = torch.tensor(pages, dtype=torch.int32, device=DEV), ints(free)
            got = B.place_tokens(table, 16, ints(lengths), ints(new), stack, ints([n_free]), n_tokens, ends=None if ends is None else ints(ends), last=last)
            results.append([*got, table, stack])
        assert all(torch.equal(a, b) for a, b in zip(*results))
        slots, starts = got.slots.tolist(), got.starts.tolist()
        assert last.tolist() == [starts[s] + k - 1 if k > 0 and starts[s] + k <= n_tokens and slots[starts[s]] >= 0 else -1 for s, k in enumerate(new)]
