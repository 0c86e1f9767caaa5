"""What the shared-key operators refuse, on the CPU: nothing is launched, so no GPU is needed."""
import ctypes as C

import pytest
import torch

import paper_2605_15609_amd as psd
from paper_2605_15609_amd import binding as B

BF = torch.bfloat16
BASE = 1 << 40       # an address that is never read


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(psd.library_path()):
        from paper_2605_15609_amd import build
        build.build()
    return psd.load_library()


def shape(**kw):
    return B._AttentionShape(**dict(dict(S=4, L=2, n_heads=8, n_kv_heads=4, d_head=64, dtype=1, ld_q=512, ld_out=512), **kw))


def seg(**kw):
    f = dict(k=BASE, vt=BASE + (1 << 30), lens=None, weights=None, stride_k=64 * 256, stride_vt=256 * 64, stride_w=0, ld_k=256, ld_vt=64, ld_w=0,
             len=50, seqs_per_unit=4, reserved=0)
    f.update(kw)
    return B._Segment(**f)


def ask(lib, sh, *segs):
    return lib.psd_attention_shared_bytes(C.byref(sh), (B._Segment * len(segs))(*segs), len(segs))


def test_the_shapes_that_are_taken(lib):
    assert ask(lib, shape(), seg()) >= 0
    assert ask(lib, shape(), seg(len=5000, ld_vt=5008), seg(seqs_per_unit=2), seg(seqs_per_unit=1)) > 0
    assert ask(lib, shape(), seg(len=0, k=None, vt=None)) >= 0
    for d in (16, 32, 64, 128):
        assert ask(lib, shape(dtype=0, d_head=d, ld_q=8 * d, ld_out=8 * d), seg(ld_k=4 * d)) >= 0
    assert lib.psd_attention_weights_bytes(C.byref(shape()), (B._Segment * 1)(seg(weights=BASE, ld_w=50)), 1) >= 0


@pytest.mark.parametrize("change", [dict(S=0), dict(L=0), dict(L=65), dict(n_heads=6), dict(n_kv_heads=0), dict(d_head=32), dict(d_head=96),
                                    dict(dtype=2), dict(ld_q=511), dict(ld_q=516), dict(ld_out=8), dict(S=1 << 30), dict(dtype=0, d_head=24)])
def test_shapes_that_are_not(lib, change):
    assert ask(lib, shape(**change), seg()) < 0
    assert B.load_library().psd_last_error()


@pytest.mark.parametrize("change", [dict(k=None), dict(vt=None), dict(k=BASE + 2), dict(vt=BASE + 8), dict(ld_k=255), dict(ld_k=260), dict(ld_vt=48),
                                    dict(ld_vt=56), dict(ld_vt=72), dict(stride_k=4), dict(stride_vt=4), dict(stride_k=-256), dict(len=-1),
                                    dict(seqs_per_unit=0), dict(seqs_per_unit=3), dict(seqs_per_unit=8), dict(reserved=1),
                                    dict(weights=BASE, ld_w=49), dict(weights=BASE, ld_w=50, stride_w=100, seqs_per_unit=1)])
def test_segments_that_are_not(lib, change):
    assert ask(lib, shape(), seg(**change)) < 0
    assert B.load_library().psd_last_error()


def test_order_and_number_of_segments(lib):
    assert ask(lib, shape(), seg(seqs_per_unit=1), seg(seqs_per_unit=4)) < 0      # fine before coarse
    assert ask(lib, shape(S=12), seg(seqs_per_unit=6), seg(seqs_per_unit=4)) < 0  # units that cross
    assert ask(lib, shape(), *[seg() for _ in range(5)]) < 0
    assert lib.psd_attention_shared_bytes(C.byref(shape()), None, 1) < 0
    assert lib.psd_attention_shared_bytes(None, (B._Segment * 1)(seg()), 1) < 0
    assert lib.psd_attention_shared_bytes(C.byref(shape()), (B._Segment * 1)(seg()), 0) < 0


def test_calls_check_pointers_and_workspace_before_anything_runs(lib):
    long = seg(len=5000, ld_vt=5008)
    s, one = shape(), (B._Segment * 1)(long)
    need = ask(lib, s, long)
    assert need > 0
    ok = dict(q=BASE, out=BASE + (1 << 20), ws=BASE, n=need)

    def call(**kw):
        a = dict(ok, **kw)
        return lib.psd_attention_shared(C.byref(s), a["q"], one, 1, a["out"], None, a["ws"], a["n"], None)
    for bad in (dict(q=None), dict(out=None), dict(q=BASE + 2), dict(out=BASE + 8), dict(ws=None), dict(ws=BASE + 128), dict(n=need - 1), dict(n=0)):
        assert call(**bad) < 0, bad
    assert lib.psd_attention_weights(C.byref(s), BASE, one, 1, None, 0, None, 0, None) < 0
    assert lib.psd_attention_weights(C.byref(s), None, one, 1, BASE, 0, None, 0, None) < 0
    assert lib.psd_attention_weights(C.byref(s), BASE, one, 1, BASE, 2, None, 0, None) < 0


def test_an_output_on_its_queries_is_refused(lib):
    one = (B._Segment * 1)(seg(len=5000, ld_vt=5008))

    def call(q, out, ld_q, ld_out):     # (without a workspace: what is not refused for its addresses is refused for that)
        assert lib.psd_attention_shared(C.byref(shape(ld_q=ld_q, ld_out=ld_out)), q, one, 1, out, None, None, 0, None) < 0
        return b"overlaps" in lib.psd_last_error()
    row = 512 * 2
    assert call(BASE, BASE, 512, 512) and call(BASE, BASE + 16, 512, 512) and call(BASE + 7 * row, BASE, 512, 512)
    assert call(BASE, BASE + row - 16, 2048, 2048) and call(BASE + row - 16, BASE, 2048, 2048) and call(BASE, BASE + row, 2048, 512)
    assert not call(BASE, BASE + 8 * row, 512, 512) and not call(BASE + 8 * row, BASE, 512, 512)
    assert not call(BASE, BASE + row, 2048, 2048) and not call(BASE + 3 * row, BASE, 2048, 2048)      # beside each other in the rows of one buffer


@pytest.mark.parametrize("heads,kv_heads,d,dtype", [(32, 32, 128, 1), (28, 4, 128, 1), (8, 8, 64, 1), (4, 4, 16, 0)])
@pytest.mark.parametrize("prefix,length", [(0, 0), (0, 480), (1024, 288), (4096, 1024), (77, 0), (16000, 4000)])
@pytest.mark.parametrize("L", [16, 32, 64])
def test_the_workspace_of_model_calls_is_enough_for_fewer_sequences(lib, heads, kv_heads, d, dtype, prefix, length, L):
    cfg = B._Config(2, heads * d, heads, kv_heads, d, 4 * heads * d, 5000, 4999, 1e-5, 0, dtype, 1.0, 32768, 1)
    S, K, up = 24, 6, lambda n: (n + 63) // 64 * 64
    kv = B._KvShared(BASE if prefix else None, BASE, BASE, BASE, prefix, prefix, max(length, 16), length, K, 0)
    kv.prefix_weights = BASE if prefix else None
    most = lib.psd_shared_workspace_bytes(C.byref(cfg), S, L, C.byref(kv)) - lib.psd_workspace_bytes(C.byref(cfg), S, L, L)
    for n in range(1, S + 1):
        for per in {1, K} if n % K == 0 else {1}:
            w = kv_heads * d
            sh = shape(S=n, L=L, n_heads=heads, n_kv_heads=kv_heads, d_head=d, dtype=dtype, ld_q=3 * heads * d, ld_out=heads * d)
            block = seg(len=L, seqs_per_unit=1, ld_k=3 * heads * d, stride_k=L * 3 * heads * d, ld_vt=up(L), stride_vt=w * up(L))
            first = [seg(len=prefix, seqs_per_unit=n, ld_k=w, ld_vt=up(prefix), weights=BASE, ld_w=prefix)] if prefix else []

            def cache(keys):
                return [seg(len=keys, seqs_per_unit=per, ld_k=w, ld_vt=up(keys), stride_k=keys * w, stride_vt=w * up(keys), weights=BASE, ld_w=keys,
                            stride_w=kv_heads * keys)] if keys else []
            sums = (n * L * heads * 4 + 255) // 256 * 256
            for segs in (first + cache(length) + [block], first + cache(length + L)):
                need = ask(lib, sh, *segs)
                weights = lib.psd_attention_weights_bytes(C.byref(sh), (B._Segment * len(segs))(*segs), len(segs))
                assert 0 <= need <= most and 0 <= weights and sums + max(need, weights if segs[-1] is block else 0) <= most, (n, per, need, weights, most)


def test_weights_of_two_segments_in_one_place_are_refused(lib):
    def call(second):      # (one that is not refused for its weights is refused for the missing lse)
        two = (B._Segment * 2)(seg(weights=BASE, ld_w=50), seg(weights=second, ld_w=50, stride_w=200, seqs_per_unit=1))
        return lib.psd_attention_weights(C.byref(shape()), BASE, two, 2, BASE, 0, None, -1, None) if second == BASE else \
            lib.psd_attention_weights(C.byref(shape()), BASE, two, 2, None, 0, None, 0, None)
    assert call(BASE) < 0 and b"same weights" in lib.psd_last_error()
    assert call(BASE + (1 << 20)) < 0 and b"same weights" not in lib.psd_last_error()


def evict(lib, src=None, dst=None, units=2, heads=4, d=64, dtype=1, keep=20, first=2, last=3, kept=BASE + (7 << 30)):
    base = dict(weights=BASE + (2 << 30), ld_w=50, stride_w=200, len=50)
    s = seg(**dict(base, **(src or {})))
    t = seg(**dict(dict(k=BASE + (4 << 30), vt=BASE + (5 << 30), weights=BASE + (6 << 30), ld_w=50, stride_w=200, len=50), **(dst or {})))
    return lib.psd_kv_evict(C.byref(s), C.byref(t), units, heads, d, dtype, keep, first, last, kept, None, None)


@pytest.mark.parametrize("change", [
    dict(keep=0), dict(keep=-1), dict(first=-1), dict(last=-1), dict(first=18, last=3), dict(first=1 << 30, last=1 << 30), dict(units=0), dict(heads=0),
    dict(d=0), dict(d=60), dict(dtype=7), dict(kept=None), dict(src=dict(weights=None)), dict(src=dict(ld_w=20)), dict(src=dict(k=None)),
    dict(dst=dict(len=19)), dict(dst=dict(lens=BASE)), dict(dst=dict(k=BASE)), dict(dst=dict(vt=BASE + (1 << 30))), dict(dst=dict(weights=BASE + (2 << 30))),
    dict(dst=dict(k=BASE + 1024)), dict(kept=BASE + 64), dict(dst=dict(stride_k=0)), dict(dst=dict(ld_vt=24)), dict(keep=1 << 30, heads=1 << 17),
])
def test_evictions_that_are_not(lib, change):
    assert evict(lib, **change) < 0
    assert lib.psd_last_error()


def test_the_binding_refuses_tensors_that_the_library_would_misread(lib):
    k, vt = torch.zeros((2, 20, 256), dtype=BF), torch.zeros((2, 256, 32), dtype=BF)
    ok = psd.KvSegment(k, vt, 64, seqs_per_unit=2)
    assert (ok.units, ok.n_kv_heads, ok.c.len, ok.c.ld_k, ok.c.ld_vt) == (2, 4, 20, 256, 32)
    for args in ((k.float(), vt), (k.half(), vt.half()), (k[0], vt), (k, vt[:1]), (k, vt[:, :128]), (k, vt[:, :, :16]), (k[..., ::2], vt[:, ::2]),
                 (k.transpose(1, 2).contiguous().transpose(1, 2), vt)):
        with pytest.raises(psd.PsdError):
            psd.KvSegment(*args, 64)
    for kw in (dict(length=21), dict(length=-1), dict(lens=torch.zeros(2)), dict(lens=torch.zeros(3, dtype=torch.int32)),
               dict(weights=torch.zeros((2, 4, 19))), dict(weights=torch.zeros((2, 3, 20))), dict(weights=torch.zeros((2, 4, 20), dtype=BF))):
        with pytest.raises(psd.PsdError):
            psd.KvSegment(k, vt, 64, **kw)
    with pytest.raises(psd.PsdError):
        psd.KvSegment(k, vt, 48)
    with pytest.raises(psd.PsdError):
        psd.KvSegments([])
    with pytest.raises(psd.PsdError):
        psd.KvSegments([ok, psd.KvSegment(k.float(), vt.float(), 64)])
    keys = psd.KvSegments([ok])
    q = torch.zeros((4, 3, 8, 64), dtype=BF)
    for bad in (q.float(), q[..., :32], q[:3], q[0], q[:, :, ::2], q.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(psd.PsdError):
            psd.psd_attention_shared(bad, keys)
    with pytest.raises(psd.PsdError):
        psd.psd_attention_shared(q, keys, lse=torch.zeros((4, 3, 8), dtype=torch.float64))
    with pytest.raises(psd.PsdError):
        psd.psd_attention_shared(q, keys, out=torch.zeros((4, 3, 8, 64)))
    with pytest.raises(psd.PsdError, match="on a GPU"):
        psd.psd_attention_shared(q, keys)
    with pytest.raises(psd.PsdError):
        psd.psd_attention_weights(q, keys, torch.zeros((4, 3, 7)))
    with pytest.raises(psd.PsdError, match="on a GPU"):
        psd.psd_attention_weights(q, keys, torch.zeros((4, 3, 8)))
    with pytest.raises(psd.PsdError, match="on a GPU"):
        psd.psd_kv_evict(ok, ok, 5)
    with pytest.raises(psd.PsdError):
        psd.psd_kv_evict(ok, ok, 0)
    with pytest.raises(psd.PsdError):
        psd.psd_kv_evict(ok, ok, 5, kept=torch.zeros((2, 4, 6), dtype=torch.int32))


@pytest.mark.parametrize("heads,kv_heads,d,dtype", [(4, 4, 128, 1), (4, 2, 128, 1), (2, 1, 64, 1), (1, 1, 64, 1), (6, 2, 16, 0)])
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 8])
def test_the_workspace_of_model_calls_is_enough_where_tiles_walk_several_units(lib, heads, kv_heads, d, dtype, K):
    # few heads: a tile of rows holds several sequences and walks the caches of all of them, so its keys can be cut into more parts than
    # the segments of one sequence have steps
    cfg = B._Config(2, heads * d, heads, kv_heads, d, 4 * heads * d, 5000, 4999, 1e-5, 0, dtype, 1.0, 32768, 1)
    w, up = kv_heads * d, lambda n: (n + 63) // 64 * 64
    for L in (16, 32, 48, 64):
        for prefix in (0, 16, 96, 500, 2000):
            for length in (0, 16, 96, 128, 700):
                for caches in (1, 2, 5):
                    S = caches * K
                    kv = B._KvShared(BASE if prefix else None, BASE, BASE if prefix else None, BASE, prefix, prefix, max(length, 16), length, K, 0)
                    most = lib.psd_shared_workspace_bytes(C.byref(cfg), S, L, C.byref(kv))
                    for n, per in {(S, K), (S, 1), (K, K), (caches, 1), (1, 1), (max(S - K, K), K)}:
                        sh = shape(S=n, L=L, n_heads=heads, n_kv_heads=kv_heads, d_head=d, dtype=dtype, ld_q=3 * heads * d, ld_out=heads * d)
                        block = seg(len=L, seqs_per_unit=1, ld_k=3 * heads * d, stride_k=L * 3 * heads * d, ld_vt=up(L), stride_vt=w * up(L))
                        first = [seg(len=prefix, seqs_per_unit=n, ld_k=w, ld_vt=up(prefix), weights=BASE, ld_w=prefix)] if prefix else []

                        def cache(keys):
                            return [seg(len=keys, seqs_per_unit=per, ld_k=w, ld_vt=up(keys), stride_k=keys * w, stride_vt=w * up(keys), weights=BASE,
                                        ld_w=keys, stride_w=kv_heads * keys)] if keys else []
                        sums = (n * L * heads * 4 + 255) // 256 * 256
                        rest = lib.psd_workspace_bytes(C.byref(cfg), n, L, L)
                        for segs in [first + cache(length) + [block]] + ([first + cache(length + L)] if per == 1 else []):
                            need = ask(lib, sh, *segs)
                            assert need >= 0
                            if segs[-1] is block:
                                weights = lib.psd_attention_weights_bytes(C.byref(sh), (B._Segment * len(segs))(*segs), len(segs))
                                need = sums + max(need, weights)
                            assert rest + need <= most, (L, prefix, length, caches, n, per, rest + need - most)


def test_outputs_on_keys_values_lengths_or_each_other_are_refused(lib):
    far = BASE + (1 << 35)

    def call(out=far, lse=far + (1 << 20), ld_out=512, **kw):     # (without a workspace: what is not refused for its addresses is refused for that)
        one = (B._Segment * 1)(seg(**dict(dict(len=5000, ld_vt=5008, stride_k=5000 * 256, stride_vt=256 * 5008, seqs_per_unit=2), **kw)))
        assert lib.psd_attention_shared(C.byref(shape(ld_out=ld_out)), BASE + (1 << 34), one, 1, out, lse, None, 0, None) < 0
        return b"lies on" in lib.psd_last_error()
    keys, values = 2 * 5000 * 512, 2 * 256 * 5008 * 2
    assert not call() and not call(lse=None)
    for at in (BASE, BASE + keys - 16, BASE + (1 << 30), BASE + (1 << 30) + values - 64):
        assert call(out=at) and call(lse=at)
    assert not call(out=BASE + keys) and not call(out=BASE + (1 << 30) + values) and not call(lse=BASE - 4 * 2 * 8 * 4) and call(lse=BASE - 4 * 2 * 8 * 4 + 4)
    assert call(lens=far) and call(lens=far + (1 << 20) + 4) and not call(lens=far - 8)
    assert call(lse=far + 7 * 1024) and call(lse=far + 8 * 1024 - 4) and not call(lse=far + 8 * 1024) and not call(lse=far - 256)
    assert call(lse=BASE + (1 << 34)) and call(lse=BASE + (1 << 34) + 8 * 1024 - 4)
    # columns of one buffer: 256 keys, 512 outputs, 256 more; and the units of a cache whose keys end in front of its values
    beside = dict(ld_k=1024, stride_k=5000 * 1024, ld_out=1024)
    assert not call(out=BASE + 512, **beside) and call(out=BASE + 496, **beside) and not call(out=BASE + 1024, **beside) and call(out=BASE + 1040, **beside)
    cache = dict(vt=BASE + keys // 2, stride_k=(keys + values) // 4, stride_vt=(keys + values) // 4)
    assert not call(**cache) and call(out=BASE + keys, **cache) and not call(out=BASE + keys + values, **cache)
    gap = dict(stride_k=5000 * 256 + 4096, stride_vt=256 * 5008 * 2)     # room for the outputs between two units
    assert not call(out=BASE + keys // 2, **gap) and call(out=BASE + keys // 2 + 16, **gap)


def test_weights_that_share_memory_are_refused(lib):
    W, Q = BASE + (1 << 36), BASE + (1 << 37)
    far, Z, S, L = W + (1 << 20), Q + (1 << 30), 64, 64

    def why(second=far, first=W, lse=Z, q=Q, prefix=dict(), cache=dict()):     # 50 shared keys, 64 caches of 40
        two = (B._Segment * 2)(seg(**dict(dict(weights=first, ld_w=50, seqs_per_unit=S), **prefix)),
                               seg(**dict(dict(weights=second, ld_w=40, stride_w=160, len=40, seqs_per_unit=1, k=BASE + (1 << 20)), **cache)))
        sh = shape(S=S, L=L)
        assert lib.psd_attention_weights_bytes(C.byref(sh), two, 2) > 0
        # (without a workspace: what is not refused for its addresses is refused for that)
        assert lib.psd_attention_weights(C.byref(sh), q, two, 2, lse, 0, None, 0, None) < 0
        return lib.psd_last_error()
    ok, shared = b"workspace of", b"same weights"
    of_prefix, of_caches, sums = 4 * 50 * 4, 64 * 160 * 4, S * L * 8 * 4
    assert ok in why() and ok in why(W + of_prefix) and ok in why(W - of_caches)
    for second in (W, W + 4, W + of_prefix - 4, W - of_caches + 4):
        assert shared in why(second)
    # columns of one buffer: [heads, 50 + 40] of a single sequence would be taken, rows of 90 that share the last column are not
    beside = dict(ld_w=90, stride_w=4 * 90)
    assert ok in why(W + 200, prefix=dict(ld_w=90), cache=beside) and shared in why(W + 196, prefix=dict(ld_w=90), cache=beside)
    for kw in (dict(lse=W), dict(lse=W + of_prefix - 4), dict(lse=far - sums + 4), dict(q=W), dict(q=far + of_caches - 16)):
        assert b"lie on q or lse" in why(**kw)
    assert ok in why(lse=W + of_prefix) and ok in why(lse=far - sums)
    for kw in (dict(prefix=dict(lens=far)), dict(prefix=dict(k=far + 64)), dict(cache=dict(lens=W + 16)), dict(cache=dict(k=W))):
        assert b"keys or lengths" in why(**kw)
    assert ok in why(prefix=dict(vt=far))      # (values are not read)


def test_destination_units_that_lie_on_each_other_are_refused(lib):
    def why(**dst):      # (what is not refused for its units is refused for `kept`, which lies on the source)
        assert evict(lib, dst=dict(dict(stride_k=20 * 256, stride_vt=256 * 64), **dst), units=3, kept=BASE) < 0
        return b"lie on each other" in lib.psd_last_error()
    assert not why()
    assert why(stride_k=0) and why(stride_k=19 * 256) and why(stride_k=20 * 256 - 8) and why(stride_k=8)
    assert why(stride_vt=0) and why(stride_vt=255 * 64) and why(stride_vt=255 * 64 + 24) and not why(stride_vt=255 * 64 + 32)      # (20 positions: slots 0 - 31)
    # beside each other: rows of three units
    assert not why(stride_k=256, ld_k=768) and why(stride_k=256, ld_k=760) and why(stride_k=248, ld_k=768) and not why(stride_k=264, ld_k=784)
    assert not why(stride_vt=64, ld_vt=192) and not why(stride_vt=32, ld_vt=96) and why(stride_vt=24, ld_vt=96) and why(stride_vt=40, ld_vt=96)


def test_evictions_whose_results_share_memory_are_refused(lib):
    P, K, far = BASE + (7 << 30), BASE + (8 << 30), BASE + (9 << 30)

    def why(kept=P, kept_lens=K, src=dict(), dst=dict(), units=2):      # (units of the destination that lie on each other are refused before anything else)
        s = seg(**dict(dict(weights=BASE + (2 << 30), ld_w=50, stride_w=200, len=50, lens=far), **src))
        t = seg(**dict(dict(k=BASE + (4 << 30), vt=BASE + (5 << 30), weights=BASE + (6 << 30), ld_w=50, stride_w=200, len=50), **dst))
        assert lib.psd_kv_evict(C.byref(s), C.byref(t), units, 4, 64, 1, 20, 2, 3, kept, kept_lens, None) < 0
        return lib.psd_last_error()
    source, each = b"overlaps the source", b"overlap each other"
    # lengths in place: other workgroups still read them
    assert source in why(kept_lens=far) and source in why(kept_lens=far + 4) and source in why(kept=far - 4 * 2 * 4 * 20 + 4)
    assert source in why(kept_lens=BASE) and source in why(kept_lens=BASE + (1 << 30)) and source in why(kept_lens=BASE + (2 << 30))
    assert each in why(kept_lens=P) and each in why(kept_lens=P + 4 * 2 * 4 * 20 - 4) and each in why(kept=BASE + (5 << 30)) and each in why(kept=BASE + (6 << 30))
    assert each in why(dst=dict(vt=BASE + (4 << 30))) and each in why(dst=dict(weights=BASE + (4 << 30))) and each in why(dst=dict(weights=P + 64))


def test_counts_near_the_end_of_32_bits_are_refused(lib):
    most = 1 << 30
    for length, taken in ((most, True), (most + 1, False), (2 ** 31 - 16, False), (2 ** 31 - 1, False)):
        long = seg(len=length, ld_vt=min(length + 15, 2 ** 31 - 1) // 16 * 16, ld_w=length, weights=BASE)
        assert (ask(lib, shape(), long) > 0) == taken
        assert (lib.psd_attention_weights_bytes(C.byref(shape(n_heads=2, n_kv_heads=2)), (B._Segment * 1)(long), 1) >= 0) == taken
    for keep in (most + 1, 2 ** 31 - 512, 2 ** 31 - 1):
        assert evict(lib, keep=keep) < 0 and b"keep" in lib.psd_last_error()


def _stub(lib):
    """What the checks of the model calls look at, of a model whose weights are in host memory."""
    import types
    shape = types.SimpleNamespace(n_layers=2, n_kv_heads=2, n_heads=2, d_head=64, vocab=100, dtype="bf16")
    return types.SimpleNamespace(shape=shape, lib=lib, handle=None, device=torch.device("cpu"), cfg=B._Config(), _tensors={"tok_emb": torch.zeros((1, 1), dtype=BF)})


def test_token_rows_that_the_library_would_misread_are_refused(lib):
    model, kv = _stub(lib), psd.SharedKv()
    good = torch.zeros((2, 64), dtype=torch.int32)
    for tokens in (good.long(), good.float(), good[0], good[None], torch.zeros((2, 128), dtype=torch.int32)[:, ::2], torch.zeros((64, 2), dtype=torch.int32).t(),
                   good.to("meta")):
        for call in (lambda: psd.psd_forward_confidence_shared(model, tokens, 0, 32, kv), lambda: psd.psd_kv_extend_shared(model, tokens, 0, 32, kv),
                     lambda: psd.psd_decode_block_shared(model, tokens, 0, 32, psd.Policy(), psd.chain_graph(2), kv)):
            with pytest.raises(psd.PsdError, match="tokens: dense int32"):
                call()


def test_caches_of_a_model_on_a_device_without_an_index(lib):
    import types
    model = _stub(lib)
    model.device = torch.device("cuda")      # (its tensors, and those of its caches, name the device that this was: here the CPU)
    s = model.shape
    cache = types.SimpleNamespace(n_seqs=2, capacity=16, model=model, mem=torch.zeros(64, dtype=torch.uint8))
    weights = torch.zeros((2, s.n_layers, s.n_kv_heads, 16))
    assert psd.SharedKv(cache=cache, length=16, cache_weights=weights).c(model, 2).cache == cache.mem.data_ptr()
    for bad in (dict(mem=torch.zeros(64, dtype=torch.uint8, device="meta")), dict(n_seqs=1), dict(model=types.SimpleNamespace(shape=types.SimpleNamespace()))):
        with pytest.raises(psd.PsdError):
            psd.SharedKv(cache=types.SimpleNamespace(**dict(vars(cache), **bad)), length=16).c(model, 2)
    with pytest.raises(psd.PsdError):
        psd.SharedKv(cache=cache, length=16, cache_weights=weights.to("meta")).c(model, 2)


def test_model_calls_run_on_the_stream_of_the_models_device(lib, monkeypatch):
    # the current device is another one: the calls have to enter the model's, and take the stream that is current there
    model, kv, seen = _stub(lib), psd.SharedKv(), []

    class Entered:
        def __init__(self, device):
            seen.append(device)

        def __enter__(self):
            raise psd.PsdError("entered")

        def __exit__(self, *what):
            pass
    monkeypatch.setattr(B, "_on_device", Entered)
    tokens = torch.zeros((2, 64), dtype=torch.int32)
    for call in (lambda: psd.psd_forward_confidence_shared(model, tokens, 0, 32, kv), lambda: psd.psd_kv_extend_shared(model, tokens, 0, 32, kv),
                 lambda: psd.psd_decode_block_shared(model, tokens, 0, 32, psd.Policy(), psd.chain_graph(2), kv)):
        with pytest.raises(psd.PsdError, match="entered"):
            call()
    assert seen == [torch.device("cpu")] * 3


def test_numbers_that_a_32_bit_argument_would_cut_are_refused(lib):
    # (1 << 32 more than a number that is taken; strides of tensors without memory)
    big = 1 << 32
    k, vt = torch.zeros((2, 20, 256), dtype=BF), torch.zeros((2, 256, 32), dtype=BF)
    with pytest.raises(psd.PsdError, match="32-bit"):
        psd.KvSegment(k, vt, 64, seqs_per_unit=big + 2)
    meta = torch.empty(1, dtype=BF, device="meta")
    with pytest.raises(psd.PsdError, match="32-bit"):
        psd.KvSegment(meta.as_strided((1, 20, 256), (0, big + 256, 1)), meta.as_strided((1, 256, 32), (0, 32, 1)), 64)
    with pytest.raises(psd.PsdError, match="32-bit"):
        psd.KvSegment(meta.as_strided((1, 20, 256), (0, 256, 1)), meta.as_strided((1, 256, 32), (0, big + 32, 1)), 64)
    one = psd.KvSegment(meta.as_strided((1, 20, 256), (0, 256, 1)), meta.as_strided((1, 256, 32), (0, 32, 1)), 64, seqs_per_unit=1 << 30)
    with pytest.raises(psd.PsdError, match="too many"):
        psd.psd_attention_weights_bytes(meta.as_strided((1 << 30, 4, 8, 64), (2048, 512, 64, 1)), psd.KvSegments([one]))
    ok = psd.KvSegment(k, vt, 64, weights=torch.zeros((2, 4, 20)))
    for args in ((big + 5, 0, 0), (5, big, 0), (5, 0, big), (5, -1, 0), (5, 0, -1), (-big + 5, 0, 0)):
        with pytest.raises(psd.PsdError) as why:
            psd.psd_kv_evict(ok, ok, *args, kept=torch.zeros((2, 4, 5), dtype=torch.int32))
        assert "on a GPU" not in str(why.value), args
    tokens = torch.zeros((2, 64), dtype=torch.int32)
    for at, length in ((big, 32), (0, big + 32), (-big, 32)):
        for call in (lambda: psd.psd_forward_confidence_shared(_stub(lib), tokens, at, length, psd.SharedKv()),
                     lambda: psd.psd_kv_extend_shared(_stub(lib), tokens, at, length, psd.SharedKv()),
                     lambda: psd.psd_decode_block_shared(_stub(lib), tokens, at, length, psd.Policy(), psd.chain_graph(2), psd.SharedKv())):
            with pytest.raises(psd.PsdError, match="32-bit"):
                call()
    for kv in (psd.SharedKv(prefix_len=big), psd.SharedKv(length=-big)):
        with pytest.raises(psd.PsdError, match="32-bit"):
            kv.c(_stub(lib), 1)


def test_launches_of_2_to_the_32_threads_are_refused(lib):
    # workgroups of 256: 2^24 of them; what is planned onto fewer is taken
    def plan(S, heads, n, ld_vt, per=1, L=1):
        s = seg(len=n, seqs_per_unit=per, ld_k=heads * 64, ld_vt=ld_vt, stride_k=n * heads * 64, stride_vt=heads * 64 * ld_vt, weights=BASE, ld_w=n, stride_w=heads * n)
        sh = shape(S=S, L=L, n_heads=heads, n_kv_heads=heads, ld_q=heads * 64, ld_out=heads * 64)
        return ask(lib, sh, s), lib.psd_attention_weights_bytes(C.byref(sh), (B._Segment * 1)(s), 1)
    attention, weights = plan((1 << 21) - 1, 8, 200, 208)        # a unit and KV head to a workgroup
    assert attention >= 0 and weights >= 0
    assert plan((1 << 20) - 1, 8, 500, 512)[1] >= 0 and plan(1 << 20, 8, 500, 512)[1] < 0      # two blocks of keys to a unit
    for S in (1 << 21, (1 << 21) + 1, 1 << 22):
        attention, weights = plan(S, 8, 200, 208)
        assert attention < 0 and weights < 0 and b"more workgroups" in lib.psd_last_error()
    assert plan(1 << 21, 8, 100, 112)[0] >= 0 and plan(1 << 23, 8, 100, 112)[0] < 0      # a unit and KV head to a wavefront
    # no keys: zeros by the kernel that joins parts, 16 rows of 64 channels a workgroup
    empty = seg(len=0, seqs_per_unit=1)
    assert ask(lib, shape(S=(1 << 24) - 1), empty) >= 0 and ask(lib, shape(S=1 << 24), empty) < 0
    # eviction: 512 threads select for a unit and KV head
    for units, heads in ((1 << 21, 4), (1 << 22, 4), (1 << 23, 1)):
        assert evict(lib, units=units, heads=heads, kept=BASE) < 0 and b"more workgroups" in lib.psd_last_error()
    assert evict(lib, units=(1 << 20) - 1, heads=4, kept=BASE) < 0 and b"more workgroups" not in lib.psd_last_error()
