"""psd_rotary on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_15609_amd as psd
from tests.gpu_common import DEV
from tests.kv8_common import rotation
from tests.shared_common import near

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rows(t, pad, shift=0):
    """t on the GPU with rows padded and begun `shift` elements into a buffer."""
    S, L, H, d = t.shape
    flat = torch.full((S * L * (H * d + pad) + shift,), float("nan"), dtype=t.dtype, device=DEV)
    v = flat[shift:].as_strided((S, L, H, d), (L * (H * d + pad), H * d + pad, d, 1))
    v.copy_(t)
    return v


def case(dtype, S, L, H, Hkv, d, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn((S, L, n, d), generator=g).to(dtype) for n in (H, Hkv))
    gains = [1 + 0.3 * torch.randn((d,), generator=g) for _ in range(2)]
    positions = torch.randint(0, 2000, (S, L), generator=g, dtype=torch.int32)
    return q, k, gains, positions


def check(q, k, freq, positions, interleaved, factor, gains, eps, got):
    for name, x, gain, y in (("q", q, gains[0], got[0]), ("k", k, gains[1], got[1])):
        want, tol = rotation(x, positions, freq, interleaved, factor, gain, eps)
        near(y, want, tol, name)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype,S,L,H,Hkv,d,rotated,pad,shift", [
    (BF, 2, 5, 8, 8, 64, 64, 0, 0), (BF, 3, 1, 28, 4, 128, 64, 8, 0), (BF, 1, 1, 1, 1, 16, 16, 0, 0), (BF, 1, 67, 32, 32, 128, 128, 0, 0),
    (F32, 2, 7, 4, 4, 16, 16, 4, 0), (F32, 2, 3, 5, 1, 96, 32, 0, 0), (BF, 2, 3, 3, 2, 256, 256, 8, 8), (BF, 2, 9, 4, 2, 80, 80, 0, 0),
    (BF, 2, 3, 3, 1, 20, 10, 1, 1), (F32, 1, 4, 3, 2, 250, 250, 3, 1), (BF, 1, 3, 2, 2, 2, 2, 0, 0), (BF, 2, 2, 4, 4, 64, 20, 0, 0), (F32, 1, 2, 2, 1, 130, 2, 0, 3)])
def test_heads_against_64_bits(dtype, S, L, H, Hkv, d, rotated, pad, shift, norm, interleaved):
    q, k, gains, positions = case(dtype, S, L, H, Hkv, d, seed=d + rotated)
    freq, _ = psd.rotary_frequencies(rotated, 10000.0)
    gains = gains if norm else [None, None]
    got = psd.psd_rotary(rows(q, pad, shift), rows(k, pad, shift), freq.to(DEV), positions=positions.to(DEV), interleaved=interleaved,
                         q_gain=gains[0] if not norm else gains[0].to(DEV), k_gain=gains[1] if not norm else gains[1].to(DEV), eps=1e-5,
                         q_out=rows(torch.zeros_like(q), pad, shift), k_out=rows(torch.zeros_like(k), pad, shift))
    check(q, k, freq, positions, interleaved, 1.0, gains, 1e-5, got)


@pytest.mark.parametrize("kind", ["plain", "linear", "base", "parts"])
@pytest.mark.parametrize("first", [0, 131072, 2 ** 31 - 70])
def test_far_positions_and_scaled_frequencies(kind, first):
    q, k, _, _ = case(F32, 2, 70, 4, 2, 64)
    freq, factor = psd.rotary_frequencies(64, 500000.0, kind, stretch=16.0, trained=8192)
    positions = (first + torch.arange(70, dtype=torch.int64)).expand(2, 70)
    got = psd.psd_rotary(q.to(DEV), k.to(DEV), freq.to(DEV), first=first, factor=factor)
    check(q, k, freq, positions, False, factor, [None, None], 1e-6, got)


def test_queries_alone_in_place_and_columns_of_one_buffer():
    q, k, gains, positions = case(BF, 3, 11, 8, 2, 64)
    freq, _ = psd.rotary_frequencies(48, 10000.0)
    alone, none = psd.psd_rotary(q.to(DEV), None, freq.to(DEV), positions=positions.to(DEV), q_gain=gains[0].to(DEV))
    assert none is None
    for interleaved in (False, True):
        buf = torch.cat([q, k, k], dim=2).to(DEV)
        views = buf[:, :, :8], buf[:, :, 8:10]
        psd.psd_rotary(*views, freq.to(DEV), positions=positions.to(DEV), q_gain=gains[0].to(DEV), interleaved=interleaved, q_out=views[0], k_out=views[1])
        check(q, k, freq, positions, interleaved, 1.0, [gains[0], None], 1e-6, views)
        assert torch.equal(buf[:, :, 10:].cpu(), k)
        if not interleaved:
            assert torch.equal(views[0], alone)
    # heads of odd width in place: the wavefront form
    q, k, gains, positions = case(BF, 3, 11, 8, 2, 30)
    freq, _ = psd.rotary_frequencies(22, 10000.0)
    buf = torch.cat([q, k], dim=2).to(DEV)
    views = buf[:, :, :8], buf[:, :, 8:]
    psd.psd_rotary(*views, freq.to(DEV), positions=positions.to(DEV), k_gain=gains[1].to(DEV), q_out=views[0], k_out=views[1])
    check(q, k, freq, positions, False, 1.0, [None, gains[1]], 1e-6, views)


def test_channels_that_are_not_turned_keep_their_bits():
    q, k, _, positions = case(BF, 2, 3, 4, 4, 64)
    q[0, 0, 0, 40], q[1, 2, 3, 63] = float("nan"), float("inf")
    freq, _ = psd.rotary_frequencies(32, 10000.0)
    for interleaved in (False, True):
        out, _ = psd.psd_rotary(q.to(DEV), k.to(DEV), freq.to(DEV), positions=positions.to(DEV), interleaved=interleaved)
        assert torch.equal(out[..., 32:].cpu().view(torch.int16), q[..., 32:].view(torch.int16))
        assert torch.isfinite(out[..., :32]).all()


def test_rows_of_zeros_with_a_norm_stay_zero():
    z = torch.zeros((1, 2, 4, 64), dtype=BF, device=DEV)
    freq = psd.rotary_frequencies(64, 10000.0)[0].to(DEV)
    out, _ = psd.psd_rotary(z, None, freq, q_gain=torch.ones(64, device=DEV))
    assert (out == 0).all()


def test_another_stream_and_a_graph():
    q, k, gains, positions = case(BF, 4, 16, 8, 2, 128)
    freq = psd.rotary_frequencies(128, 10000.0)[0]
    d = [t.to(DEV) for t in (q, k, freq, positions, gains[0], gains[1])]
    outs = torch.empty_like(d[0]), torch.empty_like(d[1])

    def call():
        psd.psd_rotary(d[0], d[1], d[2], positions=d[3], q_gain=d[4], k_gain=d[5], q_out=outs[0], k_out=outs[1])
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for i in range(3):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i
    d[3].add_(5)
    graph.replay()
    torch.cuda.synchronize()
    check(q, k, freq, positions + 5, False, 1.0, gains, 1e-6, outs)
