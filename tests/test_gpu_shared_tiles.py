"""Attention over shared keys in tiles of 128 rows: every way in which such a tile walks segments and its keys are cut, against the 64-bit
reference element by element (the bounds are derived in shared_common.Case.reference)."""
import pytest
import torch

from tests.shared_common import Case
from tests.test_gpu_shared_attention import check

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def lens(units, most):
    """Of every kind: all, one, whole tiles of 64, one more, few, none."""
    return [(most, 1, 64, 65, most - 1, 13, 0, 37)[(3 * i) % 8] for i in range(units)]


# segments in a tile's walk, whether its keys are cut, tiles of a unit and KV head at least
@pytest.mark.parametrize("H,Hkv,dh,S,L,segments,walk,cut,tiles", [
    (8, 8, 64, 8, 64, [(8, 1000, None)], 1, True, 4),
    (8, 8, 64, 8, 64, [(8, 1000, None), (2, 200, lens(4, 200)), (1, 64, None)], 3, True, 4),
    (8, 8, 64, 66, 64, [(2, 130, lens(33, 130)), (1, 64, None)], 2, False, 1),
    (2, 2, 64, 70, 64, [(2, 300, lens(35, 300))], 1, False, 1),
    (4, 1, 64, 8, 64, [(8, 4000, None), (4, 500, [500, 37]), (1, 64, None)], 3, True, 16),
    (4, 4, 128, 4, 64, [(4, 1000, None), (2, 200, [129, 200]), (1, 64, None)], 3, True, 2),
    (28, 4, 128, 8, 32, [(8, 300, [299]), (2, 100, [100, 0, 64, 3]), (1, 32, None)], 3, True, 14),      # units of 224 rows: tiles across their borders
    (10, 2, 128, 24, 32, [(24, 500, None), (2, 150, lens(12, 150)), (1, 32, None)], 3, True, 30),       # of 320 and 160
    (4, 4, 128, 72, 32, [(6, 200, lens(12, 200)), (1, 32, None)], 2, False, 2),                         # a wavefront to a sequence
    (28, 4, 128, 8, 64, [(8, 300, None), (2, 100, lens(4, 100)), (1, 64, None)], 3, False, 28),
    (28, 4, 128, 12, 48, [(12, 1000, None), (4, 200, lens(3, 200)), (1, 48, None)], 1, True, 11),       # of 336: no whole wavefronts
])
@pytest.mark.parametrize("pad", [0, 1])
def test_tiles_of_128_rows(H, Hkv, dh, S, L, segments, walk, cut, tiles, pad):
    from paper_2605_15609_amd import binding
    case = Case(BF, H, Hkv, dh, S, L, segments, seed=S + L + dh, pad=pad)
    q, keys, _ = case.device("cuda:0")
    jobs = [j for j in binding.attention_plan(q, keys) if j[2] == 1]
    print(f"[tiles] {jobs}", flush=True)
    assert any(j[1] == walk and (j[5] > 1) == cut and j[4] >= tiles for j in jobs), jobs
    check(case, weights=range(min(2, len(segments))))
