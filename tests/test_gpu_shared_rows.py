"""Attention over shared keys, row by row: what a row gets does not depend on what the other sequences of its batch hold."""
import pytest
import torch

from tests.shared_common import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float32


def put(case, s, scale):
    """Sequence s asks something else, far larger or smaller, of other keys of its own."""
    g = torch.Generator().manual_seed(1000 + s)
    case.q[s] = (scale * torch.randn(case.q[s].shape, generator=g)).to(case.dtype)
    for seg in case.segments:
        u, m = s // seg["per"], seg["held"][s // seg["per"]]
        if seg["per"] == 1:
            seg["k"][u, :m] = (scale * torch.randn(seg["k"][u, :m].shape, generator=g)).to(case.dtype)
            seg["v"][u, :m] = torch.randn(seg["v"][u, :m].shape, generator=g).to(case.dtype)


# one wavefront's 32 rows are of several sequences: rows of one unit straight from memory, a unit to a wavefront, tiles of 128 rows
@pytest.mark.parametrize("dtype,H,Hkv,dh,S,L,segments", [
    (BF, 28, 4, 128, 4, 1, [(4, 900, None)]), (BF, 8, 8, 64, 6, 5, [(6, 300, None), (1, 77, None)]), (FP, 8, 2, 32, 4, 2, [(4, 500, None), (1, 20, None)]),
    (BF, 8, 8, 64, 144, 3, [(2, 100, None)]), (BF, 4, 4, 128, 16, 16, [(16, 1000, None), (2, 200, None)]), (BF, 8, 8, 64, 48, 16, [(48, 2000, None)])])
def test_a_row_does_not_depend_on_its_neighbours(dtype, H, Hkv, dh, S, L, segments):
    import paper_2605_15609_amd as psd
    print(f"[rows] {dtype} H={H}/{Hkv} dh={dh} S={S} L={L} {segments}", flush=True)
    results = []
    for scale in (0.02, 30.0):
        case = Case(dtype, H, Hkv, dh, S, L, segments, seed=21)
        for s in range(1, S, 2):
            put(case, s, scale)
        q, keys, _ = case.device(DEV)
        lse = torch.empty(case.q.shape[:3], device=DEV)
        out = psd.psd_attention_shared(q, keys, lse=lse)
        torch.cuda.synchronize()
        results.append((out[::2].clone(), lse[::2].clone()))
    assert torch.isfinite(results[0][0]).all()
    assert all(torch.equal(a, b) for a, b in zip(*results))
