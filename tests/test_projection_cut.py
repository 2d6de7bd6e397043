"""How products with a projection in 8 bits are cut (csrc/projection_cut.h). No GPU needed."""
import random

import pytest

from cut_util import DEVICES, cuts
from test_gpu_projection_cuts import LARGE, SHAPES

QUAD = 4 * 128          # columns of the depth that parts share out


def _access(width):
    return 8 if width % 8 == 0 else 4 if width % 4 == 0 else 1


@pytest.mark.parametrize("device", DEVICES)
def test_cuts_stay_within_what_the_kernels_hold(tmp_path, device):
    rng = random.Random(5)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    asked = [(log(1, 20000), log(1, 40000), log(1, 40000)) for _ in range(4000)] + [(2 ** 31 - 256, 1, 1), (1, 2 ** 22, 2 ** 22), (65, 1, 1)]
    for (rows, width, depth), (pair, tile, parts, clusters) in zip(asked, cuts(tmp_path, asked, device)):
        quads, tiles = -(-depth // QUAD), -(-rows // tile) * -(-width // (256 if pair else 128))
        assert tile % 16 == 0 and 16 <= tile <= (224 if pair else 128) and 1 <= parts <= min(4 if pair else 8, quads)
        assert not pair or rows > 64
        fit = device[1][parts * (2 if pair else 1) - 1]
        if parts > 1:                           # a tile's parts run at the same time, all of them
            assert tiles <= fit and clusters == tiles * parts
        else:
            assert clusters == (min(tiles, fit) if pair else tiles)


@pytest.mark.parametrize("device", DEVICES)
def test_the_gpu_tests_reach_every_kernel(tmp_path, device):
    """Single CTAs and pairs, whole and with a depth that is shared, at each width of access; the highest tiles; several tiles of a pair one after the
    other. (Both directions and both types are run at each shape.)"""
    asked = [s for s in LARGE] + [(rows, n, k) for rows, k, n in SHAPES]
    reached, highest, turns = set(), {}, False
    for (rows, width, depth), (pair, tile, parts, clusters) in zip(asked, cuts(tmp_path, asked, device)):
        kind = (pair, parts > 1)
        reached.add(kind + (_access(width),))
        highest[kind] = max(highest.get(kind, 0), tile)
        turns = turns or (pair and parts == 1 and -(-rows // tile) * -(-width // 256) > 2 * clusters)
    assert reached == {(p, s, a) for p in (False, True) for s in (False, True) for a in (8, 4, 1)}
    assert highest[True, False] == 224 and highest[True, True] >= 176 and turns


def test_parts_of_a_pair(tmp_path):
    parts = {c[2] for s, c in zip(LARGE, cuts(tmp_path, LARGE)) if c[0]}
    assert parts == {1, 2, 3, 4}
