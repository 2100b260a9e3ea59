"""A model of how the 8-bit paged attention cuts its work on the device: no more pieces than its workspace and grid are planned for, whatever the lengths."""
import os
import random

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1911_02150_amd", "libmqa_decode.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built (run __graft_entry__.build())")

UNITS, SHARES, SHARES_OF_MANY, LEAST, LONGEST, LONGEST_SCALED, LOOKED_FOR = 256, 768, 512, 16, 64, 256, 1024


def block_rows(groups, R, tiles, wide):
    little = groups * tiles * R * (4 if wide > 128 else 2) <= 3 << 16 and groups * (-(-R // 16)) <= (3 if wide <= 64 else 2) * UNITS
    return 16 if R <= 16 or little else 32


def pieces(b, h_kv, blocks, tiles):
    """Of all groups; tiles: of each sequence."""
    total, longest = sum(tiles) * h_kv, max(tiles)

    def cut(into):
        per = max(1, (into + 3) // 4) * 4
        return sum(max(1, -(-t // per)) for t in tiles) * h_kv

    share = max(LEAST, -(-total // (SHARES_OF_MANY if blocks > 1 else SHARES)))
    if b > LOOKED_FOR:                       # listed by a launch of its own
        return cut(longest if longest <= LONGEST and longest * (UNITS // blocks) <= total else share)
    if b * h_kv * blocks >= UNITS and longest <= LONGEST_SCALED and longest * (UNITS // blocks) <= total:
        return cut(longest)
    most = 2 * UNITS if total * blocks > 16 * UNITS else UNITS
    while most <= 2 * UNITS:
        units = most // blocks
        if b * h_kv <= units:
            for x in range(8, 13):
                if (n := cut(-(-total * x // (8 * units)))) <= units:
                    return n
        most *= 2
    return cut(share)


LENGTHS = [lambda r, t: t, lambda r, t: r.randint(0, t), lambda r, t: r.choice([0, 1, t, r.randint(0, t)]), lambda r, t: r.choice([t, 1]), lambda r, t: min(t, int(t * r.random() ** 6))]


@pytest.mark.parametrize("seed", range(8))
def test_pieces_are_planned_for(seed):
    import paper_1911_02150_amd as m
    r, seen = random.Random(seed), 0
    for _ in range(2500):
        b = r.choice([1, 2, r.randint(1, 64), r.randint(1, 300), r.randint(1, 80), r.randint(1, 1100)])
        h_kv, R = r.choice([1, 1, 2, 4, 8, r.randint(1, 70)]), r.choice([1, 4, 8, 16, 32, 64, r.randint(1, 600), r.randint(1, 5000)])
        tiles, k = r.choice([r.randint(1, 40), r.randint(13, 300), r.randint(1, 2000)]), r.choice([32, 64, 128, 256])
        room = m.mqa_paged_scaled_decode_workspace_bytes(b, 1, R * h_kv, h_kv, 32, tiles, k, k, m.MQA_INT8)
        if not room:                         # (whole groups, or too large a call)
            continue
        seen += 1
        blocks = -(-R // block_rows(b * h_kv, R, tiles, k))
        lengths = r.choice(LENGTHS)
        n = pieces(b, h_kv, blocks, [lengths(r, tiles) for _ in range(b)])
        assert n * R * (k + 2) * 4 + b * h_kv * 8 <= room, (b, h_kv, R, tiles, k, n)
    assert seen > 500
