"""Attention over shared keys, row by row: what a row gets does not depend on what the other sequences of its batch hold, and scores may be
of any size."""
import pytest
import torch

from tests.shared_common import Case, near

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


FORMS = [(BF, 28, 4, 128, 2, 1, 300), (BF, 4, 4, 64, 3, 40, 333), (BF, 8, 8, 128, 2, 64, 200), (BF, 2, 2, 128, 2, 1, 9000), (BF, 8, 8, 64, 70, 2, 50), (FP, 4, 2, 16, 2, 3, 70),
         (FP, 2, 2, 128, 2, 20, 1500)]
LOWEST = -1.0     # times the largest number of the type


@pytest.mark.parametrize("dtype,H,Hkv,dh,S,L,n", FORMS)
@pytest.mark.parametrize("a,b", [(2.0 ** 11, 2.0 ** 12), (2.0 ** 14, 2.0 ** 14), (2.0 ** 20, 2.0 ** 20), (2.0 ** 20, -2.0 ** 20), (2.0 ** 60, 2.0 ** 60), (1.0, LOWEST), (1.0, -LOWEST)])
def test_scores_of_any_size(dtype, H, Hkv, dh, S, L, n, a, b):
    """Two sizes of scores, a b and a b (1 - 2^-7), both exact: the keys with the larger one share the row, the others draw nothing (2^16 and
    more below).  The first half of a row's keys are a segment of their own, so parts and segments meet too."""
    import paper_2605_15609_amd as psd
    if abs(b) == 1.0:
        b *= torch.finfo(dtype).max
    print(f"[rows] {dtype} H={H}/{Hkv} dh={dh} S={S} L={L} n={n} a={a:.3g} b={b:.3g}", flush=True)
    case = Case(dtype, H, Hkv, dh, S, L, [(S, n // 2, None), (1, n - n // 2, None)], seed=22)
    case.q.zero_()
    case.q[..., 0] = a
    size = torch.rand(n, generator=torch.Generator().manual_seed(23)) < 0.5
    size[:2] = torch.tensor([False, True])
    factor = torch.where(size, 1.0, 1.0 - 2.0 ** -7)
    top = size if b > 0 else ~size
    for i, s in enumerate(case.segments):
        at = slice(0, n // 2) if i == 0 else slice(n // 2, n)
        s["k"].zero_()
        s["k"][..., ::dh] = (b * factor[at]).to(dtype)[None, :, None]
    x = float(torch.tensor(a, dtype=dtype)) * float((b * factor[top][0]).to(dtype)) / dh ** 0.5
    q, keys, _ = case.device(DEV)
    lse = torch.empty(case.q.shape[:3], device=DEV)
    out = psd.psd_attention_shared(q, keys, lse=lse).double().cpu()
    lse = lse.double().cpu()
    # lse: the maximum times log2(e) / sqrt(d) and divided by log2(e), constants of their own rounding: 5 half steps, then ln of the sum
    count = int(top.sum())
    want = x + torch.log(torch.tensor(float(count), dtype=torch.float64))
    assert ((lse - want).abs() <= 5 * 2.0 ** -24 * abs(x) + 2.0 ** -20).all(), (lse - want).abs().max()
    u = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    for s in range(S):
        v = torch.cat([case.segments[0]["v"][0], case.segments[1]["v"][s]])[top].double().view(count, Hkv, dh)
        want, size_v = (t.repeat_interleave(H // Hkv, 0) for t in (v.mean(0), v.abs().mean(0)))
        # equal probabilities, each rounded to bf16 (u), n sums, the result rounded (u)
        tol = (2 * n * 2.0 ** -24 + u) * size_v + u * want.abs() + 1e-30
        assert ((out[s] - want).abs() <= tol).all(), (s, ((out[s] - want).abs() / tol).max())


@pytest.mark.parametrize("dtype,H,Hkv,dh,S,L,n", FORMS)
def test_keys_of_the_lowest_value_draw_nothing(dtype, H, Hkv, dh, S, L, n):
    import paper_2605_15609_amd as psd
    print(f"[rows] {dtype} H={H}/{Hkv} dh={dh} S={S} L={L} n={n}", flush=True)
    case = Case(dtype, H, Hkv, dh, S, L, [(S, n, None), (1, 45, None)], seed=24)
    case.q[..., 0] = case.q[..., 0].abs() + 0.5
    low = case.segments[1]["k"]
    low.zero_()
    low[..., ::dh] = torch.finfo(dtype).min
    q, keys, ws = case.device(DEV, (0, 1))
    lse = torch.empty(case.q.shape[:3], device=DEV)
    out = psd.psd_attention_shared(q, keys, lse=lse)
    psd.psd_attention_weights(q, keys, lse, accumulate=False)
    case.segments.pop()
    ref = case.reference()
    near(out, ref["out"], ref["out_tol"], "out")
    near(lse, ref["lse"], ref["lse_tol"], "lse")
    near(ws[0][..., :n], ref["w"][0], ref["w_tol"][0], "weights")
    assert (ws[1][..., :45] == 0).all()


@pytest.mark.parametrize("dtype,H,Hkv,dh,S,L,n", FORMS)
@pytest.mark.parametrize("a,b", [(2.0 ** 20, 2.0 ** 20), (2.0 ** 20, -2.0 ** 20), (1.0, LOWEST), (1.0, -LOWEST)])
def test_rows_of_huge_scores_give_no_more_than_one_each(dtype, H, Hkv, dh, S, L, n, a, b):
    """The last sequence's scores are all huge, and equal: it adds between 0 and its number of rows to a key of its own, and leaves those of
    the others alone."""
    import paper_2605_15609_amd as psd
    if abs(b) == 1.0:
        b *= torch.finfo(dtype).max
    print(f"[rows] {dtype} H={H}/{Hkv} dh={dh} S={S} L={L} n={n} a={a:.3g} b={b:.3g}", flush=True)
    case = Case(dtype, H, Hkv, dh, S, L, [(1, n, None)], seed=25)
    want = case.reference()
    case.q[-1].zero_()
    case.q[-1, ..., 0] = a
    seg = case.segments[0]
    seg["k"][-1].zero_()
    seg["k"][-1, :, ::dh] = b
    q, keys, ws = case.device(DEV, (0,))
    lse = torch.empty(case.q.shape[:3], device=DEV)
    psd.psd_attention_shared(q, keys, lse=lse)
    psd.psd_attention_weights(q, keys, lse, accumulate=False)
    got = ws[0][..., :n]
    assert torch.isfinite(got).all() and (got[-1] >= 0).all() and (got[-1] <= L * (H // Hkv)).all()
    near(got[:-1], want["w"][0][:-1], want["w_tol"][0][:-1], "weights")
