"""What the rotation and the 8-bit caches refuse, and host-only entry points, on the CPU: nothing is launched, so no GPU is needed."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2605_15609_amd as psd
from paper_2605_15609_amd import binding as B

BF = torch.bfloat16
BASE = 1 << 40       # an address that is never read
GB = 1 << 30


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(psd.library_path()):
        from paper_2605_15609_amd import build
        build.build()
    return psd.load_library()


def refused(lib, rc, *words):
    assert rc < 0
    said = lib.psd_last_error().decode()
    assert said and all(w in said for w in words), said


# ------------------------------------------------------------------------------------------------------ frequencies
def test_frequencies_are_the_formulas():
    f, one = psd.rotary_frequencies(64, 10000.0)
    j = np.arange(32)
    plain = 10000.0 ** (-2 * j / 64)
    assert one == 1.0 and np.allclose(f.numpy(), plain, rtol=1e-14)
    f, one = psd.rotary_frequencies(64, 10000.0, "linear", 4.0)
    assert one == 1.0 and np.allclose(f.numpy(), plain / 4, rtol=1e-14)
    f, one = psd.rotary_frequencies(64, 10000.0, "base", 4.0)
    assert one == 1.0 and np.isclose(f[0], 1.0) and np.isclose(f[-1], plain[-1] / 4, rtol=1e-12)
    f, factor = psd.rotary_frequencies(64, 10000.0, "parts", 4.0, trained=4096, slow=1, fast=32)
    turns = 4096 * plain / (2 * math.pi)
    assert np.isclose(factor, 0.1 * math.log(4) + 1)
    assert np.allclose(f.numpy()[turns > 32], plain[turns > 32]) and np.allclose(f.numpy()[turns < 1], plain[turns < 1] / 4)
    middle = (turns > 1) & (turns < 32)
    share = (turns[middle] - 1) / 31
    assert middle.any() and np.allclose(f.numpy()[middle], plain[middle] * (share + (1 - share) / 4), rtol=1e-13)


@pytest.mark.parametrize("args", [dict(rotated=3), dict(rotated=0), dict(rotated=-2), dict(rotated=258), dict(rotated=2 ** 33), dict(theta=0.0),
                                  dict(theta=float("nan")), dict(theta=float("inf")), dict(kind="other"), dict(kind="linear", stretch=0.5),
                                  dict(kind="linear", stretch=float("nan")), dict(kind="base", rotated=2, stretch=2.0), dict(kind="parts", stretch=2.0),
                                  dict(kind="parts", stretch=2.0, trained=4096, slow=32.0, fast=32.0), dict(kind="parts", stretch=2.0, trained=4096, slow=-1.0)])
def test_frequencies_that_are_refused(args):
    with pytest.raises(psd.PsdError):
        psd.rotary_frequencies(**{**dict(rotated=64, theta=10000.0), **args})


# --------------------------------------------------------------------------------------------------------- rotation
def rotary(lib, q=BASE, k=BASE + GB, freq=BASE + 2 * GB, positions=BASE + 3 * GB, q_gain=None, k_gain=None, q_out=BASE + 4 * GB, k_out=BASE + 5 * GB, **kw):
    f = dict(n_tokens=8, ld_q=512, ld_k=128, ld_q_out=512, ld_k_out=128, n_heads=8, n_kv_heads=2, d_head=64, rotated=64, interleaved=0, first=0, rows_per_seq=1,
             dtype=1, factor=1.0, eps=1e-6, reserved=0)
    f.update(kw)
    return lib.psd_rotary(C.byref(B._RotaryShape(**f)), q, k, freq, positions, q_gain, k_gain, q_out, k_out, None)


@pytest.mark.parametrize("change", [dict(n_tokens=0), dict(n_heads=0), dict(n_kv_heads=-1), dict(d_head=63), dict(d_head=0), dict(d_head=258), dict(rotated=0),
                                    dict(rotated=66), dict(rotated=7), dict(interleaved=2), dict(dtype=2), dict(factor=float("nan")), dict(eps=-1.0),
                                    dict(eps=float("inf")), dict(reserved=1), dict(ld_q=511), dict(ld_k=100), dict(ld_q_out=511), dict(ld_k_out=0), dict(q=None), dict(k=None),
                                    dict(freq=None), dict(q_out=None), dict(k_out=None), dict(q=BASE + 1), dict(freq=BASE + 2 * GB + 4), dict(positions=BASE + 3 * GB + 2),
                                    dict(n_tokens=1 << 50), dict(n_heads=1 << 30), dict(positions=None, rows_per_seq=0), dict(positions=None, first=-1),
                                    dict(positions=None, first=2 ** 31 - 1, rows_per_seq=2), dict(n_tokens=1 << 33, ld_q=1 << 40)])
def test_rotations_that_are_refused(lib, change):
    refused(lib, rotary(lib, **change))


def test_outputs_that_overlap(lib):
    for change in (dict(q_out=BASE + 16), dict(q_out=BASE, ld_q_out=1024), dict(q_out=BASE + GB), dict(k_out=BASE), dict(q_out=BASE + 3 * GB), dict(q_out=BASE + 2 * GB - 64),
                   dict(k_out=BASE + 4 * GB), dict(q_gain=BASE + 4 * GB + 256), dict(k_gain=BASE + 5 * GB),
                   # queries in place, keys onto columns of the queries' rows
                   dict(q_out=BASE, k_out=BASE + 128, ld_q=1024, ld_q_out=1024, ld_k_out=1024)):
        refused(lib, rotary(lib, **change), "overlap" if "gain" not in str(change) and change not in (dict(q_out=BASE + 3 * GB), dict(q_out=BASE + 2 * GB - 64)) else "lies on")


# ------------------------------------------------------------------------------------------------------------ caches
def cache(**kw):
    f = dict(codes=BASE, scales=BASE + GB, lens=None, stride_codes=2 * 128 * 128, stride_scales=2 * 4 * 2, capacity=128, len=100, block=32, format=0, n_kv_heads=2,
             d_head=64, seqs_per_unit=1, reserved=0)
    f.update(kw)
    return B._Kv8Cache(**f)


def store(lib, units=4, k=BASE + 2 * GB, v=BASE + 3 * GB, ld_k=128, ld_v=128, dtype=1, n=5, first=0, starts=None, counts=None, **kw):
    return lib.psd_kv8_store(C.byref(cache(**kw)), units, k, v, ld_k, ld_v, dtype, n, first, starts, counts, None)


def load(lib, units=4, first=0, n=5, k=BASE + 2 * GB, v=BASE + 3 * GB, ld_k=128, ld_v=128, dtype=1, **kw):
    return lib.psd_kv8_load(C.byref(cache(**kw)), units, first, n, k, v, ld_k, ld_v, dtype, None)


CACHES = [dict(codes=None), dict(scales=None), dict(codes=BASE + 8), dict(scales=BASE + GB + 4), dict(stride_codes=16392), dict(stride_scales=17), dict(stride_codes=-16),
          dict(capacity=100), dict(capacity=112), dict(capacity=-32), dict(capacity=96, block=64), dict(len=129), dict(len=-1), dict(block=8), dict(block=48),
          dict(format=2), dict(n_kv_heads=0), dict(d_head=48), dict(d_head=256), dict(reserved=1), dict(n_kv_heads=1 << 20), dict(lens=BASE + 1)]


@pytest.mark.parametrize("change", CACHES + [dict(units=0), dict(k=None), dict(v=None), dict(k=BASE + 2 * GB + 2), dict(ld_k=127), dict(ld_v=132), dict(ld_k=120), dict(dtype=3),
                                             dict(n=-1), dict(n=1 << 31 - 1), dict(first=-1), dict(first=124), dict(starts=BASE + 2), dict(counts=BASE + 4 * GB + 1),
                                             dict(stride_codes=2 * 128 * 128 - 16), dict(stride_scales=0), dict(units=1 << 24, n=128), dict(capacity=0, len=0, codes=None, scales=None)])
def test_stores_that_are_refused(lib, change):
    refused(lib, store(lib, **change))


@pytest.mark.parametrize("change", CACHES + [dict(units=0), dict(k=None), dict(v=None), dict(k=BASE + 2 * GB + 2), dict(ld_k=127), dict(ld_v=132), dict(dtype=3), dict(n=-1),
                                             dict(first=-1), dict(first=124), dict(units=1 << 24, n=128)])
def test_loads_that_are_refused(lib, change):
    refused(lib, load(lib, **change))


def test_nothing_to_do_is_done(lib):
    assert store(lib, n=0) == 0 and load(lib, n=0) == 0 and store(lib, n=0, k=None, v=None) == 0


def test_what_overlaps_is_refused(lib):
    for change in (dict(k=BASE), dict(v=BASE + GB), dict(starts=BASE + 64), dict(counts=BASE + GB + 8), dict(scales=BASE + 64), dict(lens=BASE)):
        refused(lib, store(lib, **change), "overlap")
    for change in (dict(k=BASE), dict(v=BASE + GB - 512), dict(lens=BASE + 2 * GB)):
        refused(lib, load(lib, **change), "lie on")
    refused(lib, load(lib, v=BASE + 2 * GB), "overlap")
    refused(lib, load(lib, v=BASE + 2 * GB + 128, ld_k=192, ld_v=192), "overlap")     # columns that share some


def test_more_workgroups_than_a_launch_takes(lib):
    # 2^32 threads: HIP would run the lower 32 bits of their number without an error
    big = dict(capacity=1 << 25, len=1 << 25, stride_codes=1 << 34, stride_scales=1 << 30, scales=1 << 52, k=1 << 54, v=1 << 55)
    refused(lib, load(lib, units=1 << 10, n=1 << 25, **big), "workgroups")
    refused(lib, store(lib, units=1 << 10, n=1 << 25, **big), "workgroups")


# -------------------------------------------------------------------------------------------------------- attention
def shape(**kw):
    return B._AttentionShape(**dict(dict(S=4, L=2, n_heads=8, n_kv_heads=2, d_head=64, dtype=1, ld_q=512, ld_out=512), **kw))


def attend(lib, sh=None, q=BASE + 2 * GB, k=None, v=None, ld_k=128, ld_v=128, out=BASE + 3 * GB, lse=None, ws=None, n=0, **kw):
    return lib.psd_attention_kv8(C.byref(sh or shape()), q, C.byref(cache(**kw)), k, v, ld_k, ld_v, out, lse, ws, n, None)


@pytest.mark.parametrize("change", CACHES + [dict(seqs_per_unit=0), dict(seqs_per_unit=3), dict(seqs_per_unit=8), dict(n_kv_heads=4), dict(d_head=128, capacity=64, len=10)])
def test_caches_that_attention_refuses(lib, change):
    assert lib.psd_attention_kv8_bytes(C.byref(shape()), C.byref(cache(**change)), 0) < 0
    refused(lib, attend(lib, **change))


@pytest.mark.parametrize("change", [dict(S=0), dict(L=0), dict(L=65), dict(n_heads=7), dict(n_kv_heads=0), dict(d_head=32), dict(dtype=2), dict(ld_q=511), dict(ld_q=516),
                                    dict(ld_out=8), dict(S=1 << 30)])
def test_shapes_that_attention_refuses(lib, change):
    assert lib.psd_attention_kv8_bytes(C.byref(shape(**change)), C.byref(cache()), 0) < 0
    refused(lib, attend(lib, sh=shape(**change)))


def test_calls_check_pointers_before_anything_runs(lib):
    assert lib.psd_attention_kv8_bytes(None, C.byref(cache()), 0) < 0 and lib.psd_attention_kv8_bytes(C.byref(shape()), None, 0) < 0
    assert lib.psd_attention_kv8_bytes(C.byref(shape()), C.byref(cache()), 2) < 0
    for change in (dict(q=None), dict(out=None), dict(q=BASE + 2 * GB + 2), dict(out=BASE + 3 * GB + 8), dict(k=BASE + 4 * GB), dict(v=BASE + 4 * GB),
                   dict(k=BASE + 4 * GB + 4, v=BASE + 5 * GB), dict(k=BASE + 4 * GB, v=BASE + 5 * GB, ld_k=100), dict(k=BASE + 4 * GB, v=BASE + 5 * GB, ld_v=132),
                   dict(lse=BASE + 6 * GB + 2)):
        refused(lib, attend(lib, **change))
    for change in (dict(out=BASE + 2 * GB), dict(out=BASE), dict(out=BASE + GB), dict(lse=BASE + 2 * GB), dict(lse=BASE + 3 * GB + 64), dict(lens=BASE + 3 * GB),
                   dict(k=BASE + 3 * GB, v=BASE + 5 * GB), dict(k=BASE + 4 * GB, v=BASE + 5 * GB, lse=BASE + 5 * GB)):
        refused(lib, attend(lib, **change), "lies on")


def test_forms_that_there_are_not(lib):
    for form, parts in ((-2, 0), (2, 0), (0, -1)):
        refused(lib, lib.psd_debug_force_attention_kv8(form, parts))
    try:
        plan, sh = (C.c_int32 * 4)(), shape(S=4, L=16)
        for form in (0, 1):
            for parts in (1, 2, 100):
                assert lib.psd_debug_force_attention_kv8(form, parts) == 0
                assert lib.psd_debug_attention_kv8_plan(C.byref(sh), C.byref(cache(seqs_per_unit=4)), 1, plan) == 0
                assert plan[0] == form and plan[1] == (2 if form else 8) and plan[2] == min(parts, 2 if form else 1) and plan[2] * plan[3] >= 100
    finally:
        assert lib.psd_debug_force_attention_kv8(-1, 0) == 0
    refused(lib, lib.psd_debug_attention_kv8_plan(C.byref(sh), C.byref(cache(seqs_per_unit=4)), 1, None))


def test_a_large_batch_takes_tiles_of_128_rows_and_a_small_one_of_32(lib):
    heads = dict(n_heads=32, n_kv_heads=32, d_head=128, ld_q=4096, ld_out=4096)
    for S, L, n, per, want in ((128, 64, 5120, 8, (1, 4, 1)), (16, 32, 1312, 1, (0, 1, 1)), (1, 1, 4096, 1, (0, 1, 8))):
        plan = (C.c_int32 * 4)()
        c = cache(n_kv_heads=32, d_head=128, capacity=n, len=n, stride_codes=n * 8192, stride_scales=n * 2, scales=1 << 50, seqs_per_unit=per)
        assert lib.psd_debug_attention_kv8_plan(C.byref(shape(S=S, L=L, **heads)), C.byref(c), 1, plan) == 0
        assert tuple(plan[:3]) == want and plan[2] * plan[3] >= n


def test_the_workspace_is_checked(lib):
    long = dict(capacity=1 << 20, len=1 << 20, stride_codes=1 << 33, stride_scales=1 << 30)
    need = lib.psd_attention_kv8_bytes(C.byref(shape()), C.byref(cache(**long)), 1)
    assert need > 0
    far = dict(long, q=BASE + 100 * GB, out=BASE + 101 * GB, scales=BASE + 200 * GB)
    for change in (dict(), dict(ws=BASE + 300 * GB, n=need - 1), dict(ws=BASE + 300 * GB + 128, n=need)):
        refused(lib, attend(lib, **far, **change), "workspace")


# ---------------------------------------------------------------------------------------------------------- binding
def test_a_workspace_that_lies_on_something_is_refused(lib):
    far = dict(sh=shape(S=4, L=1), capacity=32768, len=32768, lse=BASE + 5 * GB)
    need = lib.psd_attention_kv8_bytes(C.byref(far["sh"]), C.byref(cache(capacity=32768, len=32768, lens=BASE + 8 * GB)), 1)
    assert need > 0
    own = dict(k=BASE + 6 * GB, v=BASE + 7 * GB, n=need, lens=BASE + 8 * GB)
    for at in (BASE, BASE + 2 * GB, BASE + 3 * GB, BASE + 5 * GB, BASE + 6 * GB, BASE + 7 * GB, BASE + 8 * GB):
        refused(lib, attend(lib, **{**far, **own, "ws": at}), "the workspace lies on")


def test_caches_that_the_binding_refuses():
    codes, scales = torch.zeros((2, 3, 4, 2, 32 * 64), dtype=torch.uint8), torch.zeros((2, 3, 4, 2))
    c = psd.Kv8Cache(codes, scales, 64)
    assert (c.units, c.n_kv_heads, c.capacity, c.block, c.length) == (2, 3, 128, 32, 128)
    assert psd.Kv8Cache(codes, torch.zeros((2, 3, 8, 2)), 64).block == 16
    for bad in (dict(codes=codes.char()), dict(scales=scales.double()), dict(d_head=32), dict(format="fp8"), dict(length=129), dict(length=-1), dict(scales=torch.zeros((2, 3, 3, 2))),
                dict(lens=torch.zeros(2)), dict(lens=torch.zeros(3, dtype=torch.int32)), dict(codes=codes[:, :, :, :, ::2]), dict(scales=scales.transpose(0, 1)), dict(seqs_per_unit=1 << 40)):
        with pytest.raises(psd.PsdError):
            psd.Kv8Cache(**{**dict(codes=codes, scales=scales, d_head=64), **bad})
    e = psd.Kv8Cache.empty(2, 3, 64, 33, block=128, device="cpu")
    assert (e.capacity, e.block) == (128, 128)
    for bad in ((0, 3, 64, 33), (2, 3, 64, -1), (2, 3, 0, 5)):
        with pytest.raises(psd.PsdError):
            psd.Kv8Cache.empty(*bad, device="cpu")
    with pytest.raises(psd.PsdError):
        psd.Kv8Cache.empty(2, 3, 64, 33, block=8, device="cpu")


def test_rows_that_the_binding_refuses():
    c = psd.Kv8Cache.empty(2, 3, 64, 64, device="cpu")
    k = torch.zeros((2, 5, 3, 64), dtype=BF)
    for a, b in ((k.half(), k.half()), (k, k.float()), (k[:1], k[:1]), (k[..., :32], k[..., :32]), (k, k[:, :4]), (k.transpose(1, 2), k.transpose(1, 2)), (k[:, ::2].expand(2, 3, 3, 64), k)):
        with pytest.raises(psd.PsdError):
            psd.psd_kv8_store(c, a, b)
    for kw in (dict(starts=torch.zeros(3, dtype=torch.int32)), dict(counts=torch.zeros(2)), dict(first=1 << 40), dict()):    # (the last: not on a GPU)
        with pytest.raises(psd.PsdError):
            psd.psd_kv8_store(c, k, k, **kw)
    for kw in (dict(n=-1), dict(first=-(1 << 33)), dict(k_out=k), dict(n=4, k_out=k, v_out=k), dict(dtype=torch.float16), dict(n=5)):
        with pytest.raises(psd.PsdError):
            psd.psd_kv8_load(c, **kw)


def test_attention_that_the_binding_refuses():
    c = psd.Kv8Cache.empty(2, 3, 64, 64, device="cpu", seqs_per_unit=2)
    q, k = torch.zeros((4, 5, 6, 64), dtype=BF), torch.zeros((4, 5, 3, 64), dtype=BF)
    assert B.attention_kv8_plan(q, c)[0] in (0, 1)
    for args, kw in (((q[:2],), {}), ((q.half(),), {}), ((q[..., :32],), {}), ((q, k), {}), ((q, k, k[:, :4]), {}), ((q, k.float(), k.float()), {}), ((q,), dict(out=q[:, :4])),
                     ((q,), dict(lse=torch.zeros((4, 5)))), ((q.transpose(1, 2),), {}), ((q,), {})):
        with pytest.raises(psd.PsdError):
            psd.psd_attention_kv8(*((args[0], c) + args[1:]), **kw)


def test_rotations_that_the_binding_refuses():
    q, k, f = torch.zeros((2, 5, 4, 64), dtype=BF), torch.zeros((2, 5, 2, 64), dtype=BF), psd.rotary_frequencies(64, 10000.0)[0]
    for args, kw in (((q.half(), None, f), {}), ((q, k[:1], f), {}), ((q, k.float(), f), {}), ((q, k, f.float()), {}), ((q, k, f), dict(positions=torch.zeros((2, 5)))),
                     ((q, k, f), dict(positions=torch.zeros((2, 4), dtype=torch.int32))), ((q, k, f), dict(q_gain=torch.zeros(32))), ((q, k, f), dict(q_out=k)),
                     ((q, None, f), dict(k_gain=torch.zeros(64))), ((q, None, f), dict(k_out=k)), ((q, k, f), dict(first=1 << 35)), ((q, k, f[None]), {}), ((q, k, f), {})):
        with pytest.raises(psd.PsdError):
            psd.psd_rotary(*args, **kw)
