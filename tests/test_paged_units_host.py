"""How many pieces the attention over pages makes of its tiles' keys on the device, worked out here for uneven requests: the workspace has
room for them whatever the counts, the mask and the host's hints are (a piece without room would not be stored)."""
import numpy as np
import pytest

from test_paged_host import plan

FEW_ROWS, KEY_TILE = 64, 64  # rows of a request by the kernel for few, where there are both; keys of a tile


def units(new, lens, G, BQ, lo, hi, pieces, least, frame, window):
    """Units of a key head, and tiles: as the kernels count them, in 32-bit floats where they do."""
    rows = np.asarray(new, dtype=np.int64) * G
    tiles = np.where((rows < lo) | (rows > hi), 0, -(-rows // BQ))
    most = np.asarray(lens, dtype=np.int64)
    if window:
        most = np.minimum(most, window * frame + BQ + frame)
    key_tiles = -(-most // KEY_TILE)
    total = int(tiles.sum())
    if not pieces or total >= pieces:
        return total, total
    f = np.float32
    c = max(np.ceil(f((tiles.astype(f) * key_tiles.astype(f)).sum(dtype=f)) / f(pieces)), f(least))
    for _ in range(4):
        whole = int(c) if c < 1e9 else 10 ** 9
        n = int((tiles * np.maximum(1, -(-key_tiles // whole))).sum())
        if n <= pieces:
            break
        c = np.ceil(c * f(f(n) / f(pieces)))
    return n, total


@pytest.mark.parametrize("seed", range(40))
def test_room_for_every_piece(seed):
    rng = np.random.default_rng(seed)
    checked = 0
    for _ in range(150):
        R = int(np.exp(rng.uniform(0, np.log(400))))
        G, Hk, D = int(rng.choice([1, 2, 3, 5, 8, 17, 40])), int(rng.choice([1, 2, 8, 40])), int(rng.choice([64, 128]))
        top = int(np.exp(rng.uniform(0, np.log(6000))))
        new = rng.integers(0, top + 1, size=R) if rng.random() < 0.5 else np.where(rng.random(R) < 0.1, top, rng.integers(0, 3, size=R))
        new[rng.integers(0, R)] = top
        room = int(np.exp(rng.uniform(0, np.log(2 ** 31 - 65536))))
        lens = np.minimum(room, np.exp(rng.uniform(0, np.log(room + 1), size=R)).astype(np.int64))
        lens[rng.integers(0, R)] = room
        spare = int(rng.integers(0, 3))  # rows of no request
        N = int(new.sum()) + spare
        frame = int(rng.choice([0, 1, 77, 1560]))
        window = int(rng.choice([0, 1, 9])) if frame else 0
        max_q = [0, 1, top, 2 ** 31 - 1][rng.integers(0, 4)]
        max_kv = [0, 1, 300, room][rng.integers(0, 4)]
        keys = min(max_kv or room, room)
        p = plan(N, R, G * Hk, Hk, D, keys, max_q, int(rng.integers(0, 2)))
        for on, other, BQ, lo, hi, pieces, least, cap in (
                (p.few, p.big, 16 * p.few_qb, 1, FEW_ROWS if p.big else 2 ** 31 - 1, p.few_pieces, 2, p.few_cap),
                (p.big, p.few, 16 * p.big_qb * p.big_waves, FEW_ROWS + 1 if p.few else 1, 2 ** 31 - 1, p.big_pieces, 4, p.big_cap)):
            if not on or not pieces:
                continue
            n, tiles = units(new, lens, G, BQ, lo, hi, pieces, least, frame, window)
            assert n == tiles or n <= cap, (n, cap, pieces, new.tolist(), lens.tolist())
            checked += n > tiles
    assert checked
