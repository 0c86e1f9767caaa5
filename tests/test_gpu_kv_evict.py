"""Eviction of cached positions by weight: which positions stay, and that everything moves to where it belongs, to the bit."""
import math

import pytest
import torch

from tests.shared_common import kept_positions, slots

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float32


def make(dtype, Hkv, dh, units, n, seed, lens=None, ties=0, gap=0):
    g = torch.Generator().manual_seed(seed)
    k = torch.randn((units, n, Hkv * dh), generator=g).to(dtype)
    vt = torch.randn((units, Hkv * dh, (n + 15) // 16 * 16 + 16 * gap), generator=g).to(dtype)
    w = torch.rand((units, Hkv, n + 3 * gap), generator=g) ** 4
    if ties:
        w = (w * ties).floor() / ties
    return k, vt, w, lens


def run(data, Hkv, dh, keep, first, last, gap=0, with_weights=True):
    import paper_2605_15609_amd as psd
    k, vt, w, lens = data
    units, n = k.shape[0], k.shape[1]
    print(f"[evict] {k.dtype} units={units} heads={Hkv} dh={dh} n={n} lens={lens} keep={keep} first={first} last={last}", flush=True)
    on = [t.to(DEV) for t in (k, vt, w)]
    src = psd.KvSegment(on[0], on[1], dh, weights=on[2], length=n, lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV))
    dk = torch.full((units, keep + gap, Hkv * dh), 5.0, dtype=k.dtype, device=DEV)
    dvt = torch.full((units, Hkv * dh, (keep + 15) // 16 * 16 + 16 * gap), 5.0, dtype=k.dtype, device=DEV)
    dw = torch.full((units, Hkv, keep + gap), 5.0, device=DEV)
    dst = psd.KvSegment(dk, dvt, dh, weights=dw if with_weights else None)
    kept_lens = torch.empty((units,), dtype=torch.int32, device=DEV)
    kept = psd.psd_kv_evict(src, dst, keep, first=first, last=last, kept_lens=kept_lens)
    torch.cuda.synchronize()
    kept, kept_lens, dk, dvt, dw = (t.cpu() for t in (kept, kept_lens, dk, dvt, dw))
    for u in range(units):
        held = n if lens is None else min(max(lens[u], 0), n)
        m = min(held, keep)
        assert int(kept_lens[u]) == m
        assert (dk[u, m:] == 5.0).all()
        for g in range(Hkv):
            want = kept_positions(w[u, g], held, keep, first, last)
            assert kept[u, g, :m].tolist() == want and (kept[u, g, m:] == -1).all(), (u, g)
            at = slice(g * dh, (g + 1) * dh)
            assert torch.equal(dk[u, :m, at], k[u, want, at])
            assert torch.equal(dvt[u, at][:, slots(m)], vt[u, at][:, slots(n)[want]])
            rest = torch.ones(dvt.shape[2], dtype=torch.bool)
            rest[slots(m)] = False
            assert (dvt[u, at][:, rest] == 5.0).all()
            if with_weights:
                assert torch.equal(dw[u, g, :m].nan_to_num(nan=3.0), w[u, g, want].nan_to_num(nan=3.0)) and (dw[u, g, m:] == 5.0).all()
            else:
                assert (dw[u] == 5.0).all()
    return kept


@pytest.mark.parametrize("dtype,Hkv,dh", [(BF, 8, 64), (BF, 4, 128), (FP, 4, 16), (FP, 2, 128)])
@pytest.mark.parametrize("n,keep", [(1, 1), (2, 1), (17, 16), (40, 7), (64, 63), (65, 64), (300, 33), (1025, 513), (777, 777), (50, 90)])
def test_lengths(dtype, Hkv, dh, n, keep):
    run(make(dtype, Hkv, dh, 3, n, seed=n + keep), Hkv, dh, keep, min(2, keep), min(3, keep - min(2, keep)))


@pytest.mark.parametrize("ties", [1, 3, 64])
def test_ties_go_to_the_lowest_position(ties):
    run(make(BF, 4, 64, 2, 1500, seed=ties, ties=ties), 4, 64, 400, 0, 0)
    run(make(FP, 2, 32, 2, 1500, seed=ties, ties=ties), 2, 32, 1400, 5, 100)


def test_ragged_units_some_within_the_budget():
    run(make(BF, 4, 128, 6, 200, seed=3, lens=[200, 0, 1, 64, 65, 500], gap=1), 4, 128, 64, 4, 16, gap=2)
    run(make(FP, 4, 16, 3, 70, seed=4, lens=[-3, 70, 12], gap=1), 4, 16, 20, 0, 20, gap=1)


def test_weights_of_every_kind():
    data = make(BF, 1, 64, 1, 64, seed=5)
    w = data[2]
    w[0, 0, :16] = torch.tensor([0.0, -0.0, 1e-45, -1e-45, math.inf, -math.inf, math.nan, -math.nan, 1.0, -1.0, 1e38, -1e38, 0.0, -0.0, 0.5, 0.5])
    for keep in (1, 2, 10, 30, 55, 60, 62, 63):
        run(data, 1, 64, keep, 0, 0)


def test_first_and_last_positions_stay_whatever_they_drew():
    data = make(BF, 2, 64, 2, 128, seed=6)
    data[2][:, :, :10] = -math.inf
    data[2][:, :, -10:] = math.nan
    kept = run(data, 2, 64, 30, 10, 10)
    assert kept[0, 0, :10].tolist() == list(range(10)) and kept[0, 0, 20:].tolist() == list(range(118, 128))
    run(data, 2, 64, 20, 10, 10)
    run(data, 2, 64, 1, 0, 1)


def test_without_weights_in_the_destination_and_long_units():
    run(make(BF, 2, 64, 1, 5000, seed=7), 2, 64, 700, 4, 32, with_weights=False)
    run(make(FP, 1, 16, 2, 20011, seed=8, ties=512), 1, 16, 3001, 1, 1)


@pytest.mark.parametrize("dtype,Hkv,dh,units,n,keep", [
    *[(dtype, Hkv, dh, units, n, keep) for dtype, Hkv, dh, units in [(BF, 2, 64, 1), (BF, 1, 128, 3), (FP, 1, 64, 2)]
      for n, keep in [(16000, 1000), (9000, 40), (9000, 200), (8193, 8000), (4097, 129), (2049, 513)]],
    (BF, 4, 64, 70, 4097, 129), (BF, 4, 64, 70, 2049, 513), (FP, 4, 16, 64, 5000, 4500), (BF, 2, 16, 2, 32768, 600), (BF, 2, 16, 2, 32769, 9)])
def test_kept_positions_near_and_far_apart(dtype, Hkv, dh, units, n, keep):
    data = make(dtype, Hkv, dh, units, n, seed=n + keep)
    if keep == 200:      # most of them in one place, the rest all over
        data[2][:, :, 3000:3150] += 1.0
    run(data, Hkv, dh, keep, 1, 3)


def test_units_without_any_position():
    import paper_2605_15609_amd as psd
    k, vt, w = torch.ones((3, 8, 128), dtype=BF, device=DEV), torch.ones((3, 128, 16), dtype=BF, device=DEV), torch.ones((3, 2, 8), device=DEV)
    dst = [torch.full_like(t, 5.0) for t in (k, vt, w)]
    lens = torch.full((3,), 7, dtype=torch.int32, device=DEV)
    kept = psd.psd_kv_evict(psd.KvSegment(k, vt, 64, weights=w, length=0), psd.KvSegment(dst[0], dst[1], 64, weights=dst[2]), 4, 1, 1, kept_lens=lens)
    assert (kept == -1).all() and (lens == 0).all() and all((t == 5.0).all() for t in dst)


def test_other_stream_and_graph():
    import paper_2605_15609_amd as psd
    k, vt, w, _ = make(BF, 4, 64, 3, 500, seed=9)
    on = [t.to(DEV) for t in (k, vt, w)]
    src = psd.KvSegment(on[0], on[1], 64, weights=on[2])

    def room():
        return (torch.zeros((3, 100, 256), dtype=BF, device=DEV), torch.zeros((3, 256, 112), dtype=BF, device=DEV), torch.zeros((3, 4, 100), device=DEV))
    a, b = room(), room()
    want = psd.psd_kv_evict(src, psd.KvSegment(a[0], a[1], 64, weights=a[2]), 100, 4, 8)
    kept, dst = torch.zeros_like(want), psd.KvSegment(b[0], b[1], 64, weights=b[2])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        psd.psd_kv_evict(src, dst, 100, 4, 8, kept=kept)
    stream.synchronize()
    assert torch.equal(kept, want) and all(torch.equal(x, y) for x, y in zip(a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        psd.psd_kv_evict(src, dst, 100, 4, 8, kept=kept)
    for _ in range(3):
        for t in (*b, kept):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept, want) and all(torch.equal(x, y) for x, y in zip(a, b))
