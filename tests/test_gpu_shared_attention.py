"""Attention over segments of keys that a batch shares, and the weights that the keys draw, against 64-bit references.  The bounds are
derived in shared_common.Case.reference."""
import math

import numpy as np
import pytest
import torch

from tests.shared_common import Case, near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float32


def check(case, weights=(), label="", accumulate=False):
    import paper_2605_15609_amd as psd
    print(f"[shared] {label or case.__dict__.get('label', '')} {case.dtype} H={case.H}/{case.Hkv} dh={case.dh} S={case.S} L={case.L} "
          f"{[(s['per'], s['n'], s['lens']) for s in case.segments]}", flush=True)
    q, keys, ws = case.device(DEV, weights)
    lse = torch.empty(case.q.shape[:3], device=DEV)
    out = psd.psd_attention_shared(q, keys, lse=lse)
    if weights:
        psd.psd_attention_weights(q, keys, lse, accumulate=accumulate)
    torch.cuda.synchronize()
    ref = case.reference()
    worst = [near(out, ref["out"], ref["out_tol"], "out"), near(lse, ref["lse"], ref["lse_tol"], "lse")]
    for i, w in enumerate(ws):
        if w is None:
            continue
        got = w.double().cpu().numpy()
        for u, m in enumerate(case.segments[i]["held"]):
            want = ref["w"][i][u, :, :m] + (-7.0 if accumulate else 0.0)
            tol = ref["w_tol"][i][u, :, :m] + (2.0 ** -22 * 7 if accumulate else 0.0)
            worst.append(near(got[u, :, :m], want, tol, f"weights of segment {i}"))
            assert (got[u, :, m:] == -7.0).all(), "weights behind the last key were touched"
    print(f"[shared]   share of the bound: {max(worst):.3f}", flush=True)
    return out, lse, ws


SHAPES = [(BF, 8, 8, 64), (BF, 28, 4, 128), (BF, 4, 4, 128), (BF, 6, 1, 64), (FP, 4, 4, 16), (FP, 6, 2, 32), (FP, 8, 8, 64), (FP, 7, 1, 128)]


@pytest.mark.parametrize("dtype,H,Hkv,dh", SHAPES)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300])
def test_one_segment_of_every_length(dtype, H, Hkv, dh, n):
    check(Case(dtype, H, Hkv, dh, 3, 1, [(3, n, None)], seed=n), weights=(0,))


@pytest.mark.parametrize("dtype,H,Hkv,dh", SHAPES)
@pytest.mark.parametrize("L", [1, 5, 16, 33, 64])
def test_prefix_caches_and_blocks(dtype, H, Hkv, dh, L):
    check(Case(dtype, H, Hkv, dh, 6, L, [(6, 70, None), (3, 90, [90, 37]), (1, L, None)], seed=L, pad=1), weights=(0, 1))


@pytest.mark.parametrize("dtype,H,Hkv,dh", [SHAPES[1], SHAPES[6]])
def test_units_without_keys_and_rows_without_any(dtype, H, Hkv, dh):
    # sequences 0 and 2 have nothing of their own, 2 and 3 no prefix either: row 2 is empty
    out, lse, _ = check(Case(dtype, H, Hkv, dh, 4, 2, [(2, 40, [40, 0]), (1, 20, [0, 7, 0, 20])], seed=1), weights=(0, 1))
    assert (out[2] == 0).all() and torch.isneginf(lse[2]).all()
    # lengths outside the unit are cut to it
    check(Case(dtype, H, Hkv, dh, 2, 1, [(1, 40, [-5, 1000])], seed=2), weights=(0,))
    # a segment of no positions between others, and nothing at all
    check(Case(dtype, H, Hkv, dh, 2, 3, [(2, 33, None), (2, 0, None), (1, 17, None)], seed=3))
    out, lse, _ = check(Case(dtype, H, Hkv, dh, 2, 3, [(2, 0, None)], seed=4), weights=(0,))
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype,H,Hkv,dh", [SHAPES[1], SHAPES[2], SHAPES[5]])
def test_long_segments_are_cut_and_joined(dtype, H, Hkv, dh):
    check(Case(dtype, H, Hkv, dh, 2, 1, [(2, 5000, None), (1, 1237, [1237, 64])], seed=5), weights=(0, 1))
    check(Case(dtype, H, Hkv, dh, 4, 40, [(4, 1500, None), (2, 700, [3, 700]), (1, 40, None)], seed=6), weights=(0, 1))


@pytest.mark.parametrize("dtype,H,Hkv,dh,S,L", [(BF, 8, 8, 64, 70, 3), (BF, 28, 4, 128, 132, 1), (BF, 8, 8, 128, 66, 4), (FP, 8, 8, 32, 68, 2), (FP, 4, 4, 16, 131, 7)])
def test_many_units_of_few_keys(dtype, H, Hkv, dh, S, L):
    lens = [(37 * i) % 101 for i in range(S)]
    check(Case(dtype, H, Hkv, dh, S, L, [(S, 150, None), (1, 100, lens), (1, 19, None)], seed=S), weights=(1,))
    check(Case(dtype, H, Hkv, dh, S, L, [(1, 128, [128 - n for n in lens])], seed=S + 1), weights=(0,))
    check(Case(dtype, H, Hkv, dh, S, L, [(1, 1, [i % 2 for i in range(S)])], seed=S + 2))


def test_four_levels():
    check(Case(BF, 8, 2, 64, 8, 16, [(8, 130, None), (4, 65, [65, 10]), (2, 40, [1, 2, 40, 0]), (1, 16, None)], seed=7), weights=(0, 1, 2, 3))


@pytest.mark.parametrize("dtype,H,Hkv,dh", [SHAPES[1], SHAPES[6]])
def test_large_scores_and_one_key_that_takes_everything(dtype, H, Hkv, dh):
    case = Case(dtype, H, Hkv, dh, 2, 4, [(2, 200, None), (1, 50, None)], seed=8, scale=20.0)
    check(case, weights=(0, 1))


@pytest.mark.parametrize("L", [2, 20, 32, 64])
@pytest.mark.parametrize("dh", [64, 128])
def test_infinite_and_nan_keys_reach_only_those_who_see_them(L, dh):
    import paper_2605_15609_amd as psd
    case = Case(BF, 4, 4, dh, 4, L, [(4, 80, None), (1, 40, None)], seed=9)
    want = case.reference()
    case.segments[1]["k"][1, 3] = float("nan")
    case.segments[1]["vt"][2][:, 5] = float("inf")
    q, keys, _ = case.device(DEV)
    out = psd.psd_attention_shared(q, keys)
    for s in (0, 3):
        near(out[s], want["out"][s], want["out_tol"][s], f"sequence {s}")
    assert torch.isnan(out[1]).all() and not torch.isfinite(out[2]).any()


def test_a_key_of_minus_infinity_alone_in_its_tile():
    # scores of -inf (a channel of q that is positive against -inf) leave the other keys as they are
    import paper_2605_15609_amd as psd
    case = Case(FP, 2, 2, 64, 1, 1, [(1, 300, None)], seed=10)
    case.q[...] = case.q.abs()
    k = case.segments[0]["k"]
    k[:, 32:64] = 0.0
    k[:, 32:64, ::64] = -float("inf")
    gone = k.clone()
    q, keys, _ = case.device(DEV)
    lse = torch.empty(case.q.shape[:3], device=DEV)
    out = psd.psd_attention_shared(q, keys, lse=lse)
    keep = [j for j in range(300) if not 32 <= j < 64]
    x = torch.einsum("hd,nhd->hn", case.q[0, 0].double(), gone[0].view(300, 2, 64).double()[keep]) / 8.0
    p = torch.softmax(x, -1)
    o = torch.einsum("hn,nhd->hd", p, case.segments[0]["v"][0].view(300, 2, 64).double()[keep])
    assert torch.allclose(out[0, 0].double().cpu(), o, rtol=0, atol=1e-4)
    assert torch.allclose(lse[0, 0].double().cpu(), torch.logsumexp(x, -1), rtol=0, atol=1e-4)


def test_accumulated_weights_add_up():
    import paper_2605_15609_amd as psd
    case = Case(BF, 8, 4, 64, 2, 16, [(2, 100, None), (1, 33, None)], seed=11)
    check(case, weights=(0, 1), accumulate=True)
    q, keys, ws = case.device(DEV, (0,))
    lse = torch.empty(case.q.shape[:3], device=DEV)
    psd.psd_attention_shared(q, keys, lse=lse)
    psd.psd_attention_weights(q, keys, lse, accumulate=False)
    once = ws[0].clone()
    psd.psd_attention_weights(q, keys, lse)
    assert torch.equal(ws[0][..., :100], 2 * once[..., :100])
    # all weights of a row add up to 1
    case2 = Case(BF, 8, 4, 64, 2, 16, [(1, 133, None)], seed=12)
    _, _, w = check(case2, weights=(0,))
    assert abs(float(w[0][..., :133].double().sum()) - 2 * 16 * 8) < 2 * 16 * 8 * 1e-5


def test_results_do_not_depend_on_what_ran_before_and_repeat_to_the_bit():
    import paper_2605_15609_amd as psd
    case = Case(BF, 28, 4, 128, 4, 32, [(4, 600, None), (2, 200, [200, 1]), (1, 32, None)], seed=13)
    q, keys, ws = case.device(DEV, (0, 1))
    lse = torch.empty(case.q.shape[:3], device=DEV)
    work = psd.psd_attention_workspace(q, keys)
    results = []
    for fill in (0, 0xFF, 0x7F):
        work.fill_(fill)
        out = psd.psd_attention_shared(q, keys, lse=lse, ws=work)
        psd.psd_attention_weights(q, keys, lse, accumulate=False)
        results.append([out.clone(), lse.clone(), ws[0].clone(), ws[1].clone()])
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


def test_another_stream_and_a_replayed_graph():
    import paper_2605_15609_amd as psd
    case = Case(BF, 28, 4, 128, 4, 16, [(4, 300, None), (1, 100, [100, 3, 50, 17])], seed=14)
    q, keys, ws = case.device(DEV, (0, 1))
    lse = torch.empty(case.q.shape[:3], device=DEV)
    want = psd.psd_attention_shared(q, keys, lse=lse)
    psd.psd_attention_weights(q, keys, lse, accumulate=False)
    want_w = [w.clone() for w in ws]
    work, out = psd.psd_attention_workspace(q, keys), torch.zeros_like(want)
    work_w = torch.empty((256 + psd.psd_attention_weights_bytes(q, keys),), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        psd.psd_attention_shared(q, keys, out=out, lse=lse, ws=work)
    stream.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        psd.psd_attention_shared(q, keys, out=out, lse=lse, ws=work)
        psd.psd_attention_weights(q, keys, lse, accumulate=False, ws=work_w)
    for i in range(4):
        out.zero_()
        lse.zero_()
        for w in ws:
            w.fill_(-7.0)
        q.mul_(1.0)                               # the program's own work in between
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(ws, want_w)), i


@pytest.mark.parametrize("dtype,n,L", [(BF, 1, 1), (BF, 130, 64), (FP, 40, 5)])
def test_rows_that_score_minus_infinity_everywhere(dtype, n, L):
    import paper_2605_15609_amd as psd
    S, H, dh = 2, 4, 64
    q = torch.rand((S, L, H, dh), generator=torch.Generator().manual_seed(n)).to(dtype).to(DEV) + 0.5
    k, vt = torch.full((S, n, H * dh), -math.inf, dtype=dtype, device=DEV), torch.ones((S, H * dh, (n + 15) // 16 * 16), dtype=dtype, device=DEV)
    k[1] = 1.0        # the second sequence's keys are ordinary ones
    w, lse = torch.full((S, H, n), 0.25, device=DEV), torch.empty((S, L, H), device=DEV)
    keys = psd.KvSegments([psd.KvSegment(k, vt, dh, weights=w)])
    out = psd.psd_attention_shared(q, keys, lse=lse)
    psd.psd_attention_weights(q, keys, lse)
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all() and (w[0] == 0.25).all()
    # the same values everywhere, so out is a sum of n equal terms over their sum: n - 1 additions each and a division, half a step apiece
    assert (out[1].double() - 1).abs().max() <= 2 * n * 2.0 ** -24 and torch.isfinite(lse[1]).all()
    assert abs(float(w[1].double().sum()) - (0.25 * n + L) * H) < 1e-4 * n * L * H


@pytest.mark.parametrize("shape", [(BF, 8, 8, 64, 4, 1), (BF, 28, 4, 128, 4, 32), (FP, 4, 2, 16, 2, 5)])
def test_a_replayed_graph_follows_the_lengths_in_memory(shape):
    import paper_2605_15609_amd as psd
    dtype, H, Hkv, dh, S, L = shape
    case = Case(dtype, H, Hkv, dh, S, L, [(S, 700, [700]), (1, 200, [200] * S)], seed=15)
    q, keys, ws = case.device(DEV, (0, 1))
    lens = [s.lens for s in keys.segments]
    lse, out, work = torch.empty(case.q.shape[:3], device=DEV), torch.zeros_like(q), psd.psd_attention_workspace(q, keys)
    work_w = torch.empty((256 + psd.psd_attention_weights_bytes(q, keys),), dtype=torch.uint8, device=DEV)

    def step():
        psd.psd_attention_shared(q, keys, out=out, lse=lse, ws=work)
        psd.psd_attention_weights(q, keys, lse, accumulate=False, ws=work_w)
    step()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for a, b in ((700, 200), (0, 3), (65, 0), (0, 0), (699, 128)):
        lens[0].fill_(a)
        lens[1].copy_(torch.tensor([max(b - i, 0) for i in range(S)], dtype=torch.int32))
        results = []
        for run in (step, graph.replay):
            for t in (out, lse, *ws):
                t.fill_(5.0)
            run()
            torch.cuda.synchronize()
            results.append([t.clone() for t in (out, lse, *ws)])
        assert all(torch.equal(x, y) for x, y in zip(*results)), (a, b)
        if a == 0 and b == 0:
            assert (results[0][0] == 0).all() and torch.isneginf(results[0][1]).all() and (results[0][2] == 5.0).all()


def test_calls_at_the_same_time_on_two_streams():
    import paper_2605_15609_amd as psd
    cases = [Case(BF, 28, 4, 128, 8, 32, [(8, 2000, None), (1, 300, None)], seed=16), Case(BF, 28, 4, 128, 8, 1, [(8, 5000, None), (1, 77, None)], seed=17)]
    held = []
    for case in cases:
        q, keys, _ = case.device(DEV, ())
        held.append((q, keys, psd.psd_attention_shared(q, keys), torch.empty_like(q), psd.psd_attention_workspace(q, keys), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for q, keys, _, out, work, stream in held:
            with torch.cuda.stream(stream):
                psd.psd_attention_shared(q, keys, out=out, ws=work)
    torch.cuda.synchronize()
    for _, _, want, out, _, _ in held:
        assert torch.equal(out, want)


def test_offsets_beyond_32_bits():
    import paper_2605_15609_amd as psd
    n, dh, ld_k, ld_vt = 2100, 128, 1 << 20, 1 << 24
    case = Case(BF, 4, 1, dh, 2, 3, [(2, n, None)], seed=15)
    seg = case.segments[0]
    big_k = torch.empty((n * ld_k,), dtype=BF, device=DEV)
    k = big_k.as_strided((1, n, dh), (0, ld_k, 1))
    k.copy_(seg["k"][:, :n].to(DEV))
    big_v = torch.empty((dh * ld_vt,), dtype=BF, device=DEV)
    vt = big_v.as_strided((1, dh, seg["vt"].shape[2]), (0, ld_vt, 1))
    vt.copy_(seg["vt"].to(DEV))
    assert n * ld_k * 2 > 1 << 32 and dh * ld_vt * 2 >= 1 << 32
    w = torch.zeros((1, 1, n), device=DEV)
    keys = psd.KvSegments([psd.KvSegment(k, vt, dh, seqs_per_unit=2, weights=w)])
    q = case.q.to(DEV)
    lse = torch.empty(case.q.shape[:3], device=DEV)
    out = psd.psd_attention_shared(q, keys, lse=lse)
    psd.psd_attention_weights(q, keys, lse, accumulate=False)
    ref = case.reference()
    near(out, ref["out"], ref["out_tol"], "out")
    near(w, ref["w"][0], ref["w_tol"][0], "weights")


def test_out_of_padded_rows_leaves_the_padding():
    import paper_2605_15609_amd as psd
    case = Case(BF, 4, 2, 64, 3, 5, [(3, 50, None)], seed=16)
    q, keys, _ = case.device(DEV)
    wide = torch.full((3, 5, 4 * 64 + 16), 9.0, dtype=BF, device=DEV)
    out = wide.as_strided((3, 5, 4, 64), (wide.stride(0), wide.stride(1), 64, 1))
    psd.psd_attention_shared(q, keys, out=out)
    ref = case.reference()
    near(out, ref["out"], ref["out_tol"], "out")
    assert (wide[..., 256:] == 9.0).all()
