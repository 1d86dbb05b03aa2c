"""Where token_scan keeps the factors of a chunk: the index arithmetic of the kernels, restated (no GPU needed).

The lengths of the sequences lie on the device, so the host sizes the workspace from (n_tokens, n_seqs) alone and each kernel
works out a chunk's place by itself.  Whatever the offsets hold, each chunk then has a place of its own inside the workspace,
and the parts that a long sequence is cut into, likewise.
"""
import numpy as np
import pytest

C = 64


def clamped(cu, n_tokens, s):
    """token_range: offsets that leave the buffer or run backwards give shorter or empty sequences."""
    start = min(max(int(cu[s]), 0), n_tokens)
    stop = min(max(int(cu[s + 1]), start), n_tokens)
    return start, stop - start


def ceil_div(a, b):
    return -(-a // b)


def lengths(rng, n_seqs, top):
    kind = rng.integers(4)
    if kind == 0:
        return rng.integers(0, 3, n_seqs)
    if kind == 1:
        return rng.integers(0, top, n_seqs)
    if kind == 2:
        return C * rng.integers(0, 5, n_seqs) + rng.integers(-1, 2, n_seqs).clip(0)
    return np.where(rng.random(n_seqs) < 0.9, 0, top)


@pytest.mark.parametrize("seed", range(40))
def test_each_chunk_has_its_own_place(seed):
    rng = np.random.default_rng(seed)
    n_seqs = int(rng.integers(1, 50))
    cu = np.concatenate([[0], lengths(rng, n_seqs, int(rng.choice([64, 200, 1500]))).cumsum()])
    n_tokens = int(cu[-1]) + int(rng.integers(0, 100))           # rows behind the last sequence
    places = n_tokens // C + n_seqs
    taken = set()
    for s in range(n_seqs):
        start, n = clamped(cu, n_tokens, s)
        for c in range(ceil_div(n, C)):
            place = start // C + s + c
            assert 0 <= place < places and place not in taken
            taken.add(place)


@pytest.mark.parametrize("seed", range(40))
def test_places_stay_inside_whatever_the_offsets_hold(seed):
    rng = np.random.default_rng(seed)
    n_seqs, n_tokens = int(rng.integers(1, 30)), int(rng.integers(1, 3000))
    cu = rng.integers(-5000, 8000, n_seqs + 1)
    cu[rng.integers(n_seqs + 1)] = rng.choice([-2 ** 31, 2 ** 31 - 1])
    for s in range(n_seqs):
        start, n = clamped(cu, n_tokens, s)
        assert 0 <= start and n >= 0 and start + n <= n_tokens
        if n:
            assert start // C + s + ceil_div(n, C) - 1 < n_tokens // C + n_seqs


def seq_of(cu, n_tokens, n_seqs, x, unit):
    """token_seq_of: the last sequence whose places start at x or before, 32 candidates at a time."""
    lo, n = 0, n_seqs
    while n > 1:
        step = ceil_div(n, 32)
        k = 0
        for lane in range(32):
            s = lo + lane * step
            if s < lo + n and clamped(cu, n_tokens, s)[0] // unit + s <= x:
                k = lane
        n = min(step, lo + n - (lo + k * step))
        lo += k * step
    return lo


@pytest.mark.parametrize("unit", [4, 64, 1920])
@pytest.mark.parametrize("seed", range(10))
def test_a_place_finds_its_sequence(seed, unit):
    rng = np.random.default_rng(seed)
    n_seqs = int(rng.choice([1, 2, 31, 32, 33, 90, 1100]))
    cu = np.concatenate([[0], lengths(rng, n_seqs, 4 * unit).cumsum()])
    n_tokens = int(cu[-1]) + int(rng.integers(0, 100))
    found = {}
    for x in range(n_tokens // unit + n_seqs):
        s = seq_of(cu, n_tokens, n_seqs, x, unit)
        assert 0 <= s < n_seqs
        start, n = clamped(cu, n_tokens, s)
        piece = x - (start // unit + s)
        if 0 <= piece < ceil_div(n, unit):
            assert (s, piece) not in found
            found[s, piece] = x
    # nothing is left out
    assert len(found) == sum(ceil_div(clamped(cu, n_tokens, s)[1], unit) for s in range(n_seqs))
