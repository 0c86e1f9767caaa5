"""8-bit caches on the GPU: what is stored and read back, exactly, and attention over it against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_15609_amd as psd
from paper_2605_15609_amd import binding as B
from tests.gpu_common import DEV, say
from tests.kv8_common import Cache, attention, spots, stored, table
from tests.shared_common import near

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rows(t, pad):
    a, n, h, d = t.shape
    flat = torch.full((a, n, h * d + pad), float("nan"), dtype=t.dtype, device=DEV)
    flat[..., :h * d] = t.reshape(a, n, h * d).to(DEV)
    return flat.as_strided(t.shape, (flat.stride(0), flat.stride(1), d, 1))


def numbers(cache):
    """codes as numbers [units, heads, positions, d] (keys, values) and scales of a cache on the GPU."""
    t = table(cache.format)
    flat = cache.codes.cpu().numpy().reshape(cache.units, cache.n_kv_heads, -1)
    s = cache.scales.cpu().numpy()
    return [t[flat[:, :, a]] for a in spots(cache.capacity, cache.d_head)], [s[..., 0], s[..., 1]]


def same(a, b):
    return ((a == b) | (np.isnan(a) & np.isnan(b))).all()


def check_store(host, dev, k, v, starts, counts, pad=0, call={}):
    want, scales = stored(host, k.double().numpy(), v.double().numpy(), starts, counts)
    psd.psd_kv8_store(dev, rows(k, pad), rows(v, pad), **call)
    torch.cuda.synchronize()
    got, got_scales = numbers(dev)
    for i in (0, 1):
        assert same(got_scales[i], scales[i]), f"scales {i}"
        # behind the last new row of a block codes stand for nothing
        for u in range(host.units):
            end = starts[u] + counts[u]
            for lo, hi in ((0, end), (-(-end // host.block) * host.block, host.n)):
                assert same(got[i][u, :, max(lo, 0):hi], want[i][u, :, max(lo, 0):hi]), f"codes {i} of unit {u}"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,units,Hkv,d,positions,block,n,starts,counts,pad", [
    (BF, 2, 4, 64, 96, 32, 96, [0, 0], None, 0), (BF, 3, 2, 128, 300, 32, 70, [31, 32, 222], None, 8), (F32, 3, 4, 64, 400, 16, 48, [333, 340, 351], None, 4),
    (F32, 2, 3, 16, 64, 16, 1, [15, 16], None, 0), (BF, 2, 2, 32, 256, 128, 200, [5, 60], [200, 0], 0), (BF, 4, 1, 128, 512, 64, 65, [-3, 500, 600, 63], [65, 65, 65, 1], 0),
    (F32, 1, 1, 128, 128, 128, 128, [0], None, 0), (BF, 1, 32, 128, 1024, 32, 1024, [0], None, 0), (BF, 2, 2, 64, 64, 16, 30, [1, 17], [30, 99], 0),
    (BF, 2, 2, 64, 64, 16, 16, [16, 32], [16, -4], 0)])
def test_codes_and_scales_are_exact(fmt, dtype, units, Hkv, d, positions, block, n, starts, counts, pad):
    host = Cache(units, Hkv, d, positions, block, fmt, seed=n)
    g = torch.Generator().manual_seed(n + d)
    # magnitudes from one row to the next so that some blocks grow and some do not
    size = 2.0 ** (3 * torch.randn((units, n, 1, 1), generator=g)) * 0.3
    k, v = ((size * torch.randn((units, n, Hkv, d), generator=g)).to(dtype) for _ in range(2))
    dev = host.device(DEV, pad=3)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    held = [min(max(c, 0), n) for c in counts] if counts else [n] * units
    check_store(host, dev, k, v, starts, held, pad, dict(starts=ints(starts), counts=ints(counts) if counts else None))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_quotients_on_and_next_to_borders(fmt, dtype):
    """Rows whose quotients by the scale lie on a border between two codes or one step of the type beside it."""
    t = np.unique(table(fmt)[np.isfinite(table(fmt))])
    t = t[np.abs(t) <= (127 if fmt == "int8" else 448)]
    middle = ((t[1:] + t[:-1]) / 2).astype(np.float64)
    host = Cache(1, 1, 128, 32, 32, fmt)
    for scale in (1.0, 0.0371, 2.0 ** -99, 2.0 ** -130, 3e35):
        s = np.float32(np.float32(scale) * t[-1]) / np.float64(t[-1])
        base = torch.from_numpy((middle * s)).to(dtype)
        x = torch.cat([base, torch.nextafter(base.float(), torch.full_like(base.float(), 1e38)).to(dtype),
                       torch.nextafter(base.float(), torch.full_like(base.float(), -1e38)).to(dtype)])
        x = x[torch.randperm(len(x), generator=torch.Generator().manual_seed(1))][:4095]
        x = torch.cat([x, torch.zeros(4095 - len(x), dtype=dtype), torch.tensor([float(np.float32(s * t[-1]))]).to(dtype)])
        k = x.view(1, 32, 1, 128)
        check_store(host, host.device(DEV), k, k.flip(1), [0], [32])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_blocks_of_zeros_and_blocks_without_a_value(fmt):
    host = Cache(1, 2, 64, 128, 32, fmt)
    k, v = (torch.randn((1, 128, 2, 64), generator=torch.Generator().manual_seed(3)).to(BF) for _ in range(2))
    k[0, :32] = 0
    k[0, 40, 0, 5], v[0, 70, 1, 6] = float("nan"), float("-inf")
    k[0, 96:] = 2.0 ** -133        # scales below the smallest normal number, or none
    dev = host.device(DEV)
    check_store(host, dev, k, v, [0], [128])
    a, b = psd.psd_kv8_load(dev, dtype=F32)
    a, b = a.cpu(), b.cpu()
    assert (a[0, :32] == 0).all() and torch.isnan(a[0, 32:64, 0]).all() and torch.isfinite(a[0, 32:64, 1]).all() and torch.isfinite(a[0, 64:]).all()
    assert torch.isnan(b[0, 64:96, 1]).all() and torch.isfinite(b[0, 64:96, 0]).all()
    # rows behind it in the block cannot bring it back; begun anew it is read again
    good = torch.ones((1, 8, 2, 64), dtype=BF, device=DEV)
    psd.psd_kv8_store(dev, good, good, first=48)
    assert torch.isnan(psd.psd_kv8_load(dev, dtype=F32)[0][0, 32:64, 0]).all()
    psd.psd_kv8_store(dev, good, good, first=32)
    assert (psd.psd_kv8_load(dev, 32, 8)[0].float() == 1).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_is_read_back_is_rounded_once(fmt, dtype):
    host = Cache(3, 2, 64, 150, 32, fmt, lens=[150, 77, 0], seed=5)
    dev = host.device(DEV)
    for first, n in ((0, 150), (33, 64), (64, 13), (149, 1), (31, 2)):
        k, v = (rows(torch.full((3, n, 2, 64), -7.0, dtype=dtype), 8) for _ in range(2))
        psd.psd_kv8_load(dev, first, n, k_out=k, v_out=v)
        for u in range(3):
            m = max(0, min(host.held[u] - first, n))
            for got, want in zip((k, v), host.read(u)):
                assert torch.equal(got[u, :m].cpu(), torch.from_numpy(want[first:first + m].copy()).to(dtype))
                assert (got[u, m:] == -7.0).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_every_width_and_block_there_and_back(fmt, dtype, d, block):
    """Rows that begin and end inside blocks: codes and scales, and what is read back, exactly."""
    host = Cache(3, 3, d, 290, block, fmt, seed=block + d)
    dev = host.device(DEV, length=host.n)
    g = torch.Generator().manual_seed(block * d)
    k, v = ((2.0 ** torch.randn((3, 150, 1, 1), generator=g) * torch.randn((3, 150, 3, d), generator=g)).to(dtype) for _ in range(2))
    starts, counts = [0, 37, 128], [150, 149, 131]
    number, scales = stored(host, k.double().numpy(), v.double().numpy(), starts, counts)
    check_store(host, dev, k, v, starts, counts, pad=8, call=dict(starts=torch.tensor(starts, dtype=torch.int32, device=DEV),
                                                                  counts=torch.tensor(counts, dtype=torch.int32, device=DEV)))
    got = psd.psd_kv8_load(dev, 3, 180, dtype=dtype)
    for u in range(3):
        held = range(max(starts[u], 3), min(starts[u] + counts[u], 183))
        at = np.array(held)
        for i in (0, 1):
            want = number[i][u][:, at] * scales[i][u].astype(np.float64)[:, at // block, None]
            assert torch.equal(got[i][u, at - 3].cpu(), torch.from_numpy(np.swapaxes(want, 0, 1).copy()).to(dtype)), (u, i)


def test_token_by_token_is_the_same_as_rules_say():
    """One token at a time: a block's scale grows step by step, and what it holds is rounded again each time."""
    host = Cache(2, 2, 64, 64, 32, "int8")
    dev = host.device(DEV)
    g = torch.Generator().manual_seed(9)
    for i in range(40):
        k, v = ((0.1 * (1 + i) * torch.randn((2, 1, 2, 64), generator=g)).to(BF) for _ in range(2))
        starts = [i, i + 7]
        number, scales = stored(host, k.double().numpy(), v.double().numpy(), starts, [1, 1])
        psd.psd_kv8_store(dev, k.to(DEV), v.to(DEV), starts=torch.tensor(starts, dtype=torch.int32, device=DEV))
        host.codes, host.scales = dev.codes.cpu().numpy(), dev.scales.cpu().numpy()
        got, got_scales = numbers(dev)
        for j in (0, 1):
            assert same(got_scales[j], scales[j])
            for u in range(2):
                assert same(got[j][u, :, :starts[u] + 1], number[j][u, :, :starts[u] + 1]), (i, j, u)


# ----------------------------------------------------------------------------------------------------------- attention
@pytest.fixture
def forced():
    """Forces the form and the parts of the calls of a test."""
    lib = psd.load_library()
    yield lambda form, parts=0: B._check(lib.psd_debug_force_attention_kv8(form, parts))
    lib.psd_debug_force_attention_kv8(-1, 0)


def run_attention(dtype, H, Hkv, d, S, L, per, positions, block, fmt, lens, own, pad=0, seed=0, scale=1.5):
    g = torch.Generator().manual_seed(seed)
    q = (scale * torch.randn((S, L, H, d), generator=g)).to(dtype)
    host = Cache(S // per, Hkv, d, positions, block, fmt, seed=seed, lens=lens)
    k, v = (torch.randn((S, L, Hkv, d), generator=g).to(dtype) if own else None for _ in range(2))
    want = attention(q, host, per, k, v)
    cache = host.device(DEV, per=per, pad=pad)
    dq, dk, dv = (None if t is None else rows(t, 8 * pad) for t in (q, k, v))
    out, lse = rows(torch.zeros_like(q), 8 * pad), torch.empty((S, L, H), dtype=F32, device=DEV)
    psd.psd_attention_kv8(dq, cache, dk, dv, out=out, lse=lse)
    torch.cuda.synchronize()
    plan = B.attention_kv8_plan(dq, cache, own)
    a, b = near(out, want["out"], want["out_tol"], "out"), near(lse, want["lse"], want["lse_tol"], "lse")
    say(f"plan {plan}, {a:.3f} and {b:.3f} of the bounds")
    return plan


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,H,Hkv,d,S,L,per,positions,block,lens,own,pad", [
    (BF, 8, 8, 64, 4, 1, 1, 300, 32, [300, 1, 33, 64], True, 0),            # single rows
    (BF, 28, 4, 128, 3, 1, 1, 700, 32, [0, 699, 31], False, 1),             # a unit without a position
    (BF, 28, 4, 128, 2, 1, 1, 5000, 16, [5000, 129], True, 0),              # parts, few rows
    (BF, 4, 4, 128, 2, 32, 1, 95, 64, None, True, 1),                       # one tile of rows exactly
    (BF, 8, 2, 64, 6, 5, 3, 77, 128, [77, 40], True, 0),                    # tiles with rows of several sequences, few rows
    (BF, 8, 2, 64, 12, 13, 6, 333, 32, [333, 200], True, 1),                # the same, many rows: 312 of 128 at a time
    (BF, 8, 1, 128, 4, 37, 2, 130, 32, [1, 130], False, 0),                 # many rows
    (BF, 28, 4, 128, 6, 64, 3, 2100, 32, [2100, 1000], True, 0),            # many rows, parts
    (BF, 4, 1, 64, 1, 16, 1, 64, 32, None, False, 0),                       # 64 rows: the smallest of the second form
    (BF, 4, 2, 128, 2, 33, 1, 0, 32, None, True, 0),                        # no cache, more rows than a step of keys
    (F32, 4, 4, 16, 3, 16, 1, 100, 16, [100, 7, 16], True, 1),
    (F32, 4, 2, 32, 4, 3, 2, 65, 32, [65, 1], True, 0),
    (F32, 8, 8, 64, 3, 16, 1, 410, 64, [410, 3, 64], True, 0),
    (F32, 2, 1, 128, 2, 64, 1, 900, 32, None, True, 0)])                    # parts in fp32
def test_attention_against_64_bits(forced, fmt, dtype, H, Hkv, d, S, L, per, positions, block, lens, own, pad):
    for form in (-1, 0, 1) if dtype == BF else (-1,):
        for parts in (0, 3) if form >= 0 else (0,):
            forced(form, parts)
            plan = run_attention(dtype, H, Hkv, d, S, L, per, positions, block, fmt, lens, own, pad, seed=positions + L)
            assert form < 0 or plan[0] == form
            assert parts == 0 or plan[2] == min(parts, -(-(positions or 1) // (64 if form else 128))) or plan[2] == 2


@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_a_unit_without_a_position_gives_zeros(forced, form, parts):
    forced(form, parts)
    host = Cache(2, 2, 64, 64, 32, "int8", lens=[0, 64])
    q = torch.randn((2, 3, 4, 64)).to(BF).to(DEV)
    lse = torch.empty((2, 3, 4), device=DEV)
    out = psd.psd_attention_kv8(q, host.device(DEV), lse=lse)
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all() and torch.isfinite(lse[1]).all()
    empty = psd.Kv8Cache(torch.empty((2, 2, 0, 2, 2048), dtype=torch.uint8, device=DEV), torch.empty((2, 2, 0, 2), device=DEV), 64)
    out = psd.psd_attention_kv8(q, empty, lse=lse)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("L,group", [(1, 1), (5, 3), (16, 2), (64, 4)])
@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_a_draft_without_a_value_leaves_the_others_alone(forced, form, parts, L, group):
    """Sequences that share a cache: NaN in one's own block reaches none of the others, whatever tile their rows share."""
    forced(form, parts)
    S, H, Hkv, d = 6, group, 1, 64
    g = torch.Generator().manual_seed(L)
    q, host = torch.randn((S, L, H, d), generator=g).to(BF).to(DEV), Cache(2, Hkv, d, 45, 32, "e4m3")
    k, v = (torch.randn((S, L, Hkv, d), generator=g).to(BF).to(DEV) for _ in range(2))
    cache = host.device(DEV, per=3)
    good = psd.psd_attention_kv8(q, cache, k, v)
    for bad in (float("nan"), float("inf")):
        v2, k2 = v.clone(), k.clone()
        v2[4, L // 2, 0, 7] = bad
        k2[1, 0, 0, 9] = float("nan")
        got = psd.psd_attention_kv8(q, cache, k2, v2)
        for s in (0, 2, 3, 5):
            assert torch.equal(got[s], good[s]), s
        assert torch.isnan(got[1]).all() and not torch.isfinite(got[4][..., 7]).any() and torch.isfinite(got[4][..., 8]).all()


@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_a_cache_block_without_a_value_reaches_who_sees_it(forced, form, parts):
    forced(form, parts)
    host = Cache(2, 1, 64, 100, 32, "int8")
    host.scales[1, 0, 1, 0] = np.nan
    q = torch.randn((2, 2, 2, 64)).to(BF).to(DEV)
    out = psd.psd_attention_kv8(q, host.device(DEV))
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1]).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("L", [4, 64])
@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_scores_of_any_size(forced, form, parts, fmt, L):
    """Keys of the same code at scales that make scores up to 2^30: the largest ones share the weight, none of the sums overflows."""
    forced(form, parts)
    d, n = 64, 160
    host = Cache(1, 1, d, n, 32, fmt)
    for exponent in (4, 12, 20, 24):
        code = 100 if fmt == "int8" else 0x74       # 100 and 192
        host.codes[0, 0, :, 0] = code
        host.scales[0, 0, :, 0] = 2.0 ** exponent
        host.scales[0, 0, 2, 0] = 2.0 ** (exponent + 1)
        q = torch.ones((1, L, 1, d), dtype=BF)
        for sign in (1, -1):
            lse = torch.empty((1, L, 1), device=DEV)
            out = psd.psd_attention_kv8((sign * q).to(DEV), host.device(DEV), lse=lse)
            assert torch.isfinite(out).all() and torch.isfinite(lse).all()
            values = host.read(0)[1][:, 0]
            top = values[64:96] if sign > 0 else np.concatenate([values[:64], values[96:]])
            # equal probabilities over the largest: half a bf16 step of each, and of the result; sums of 160 in fp32
            tol = (2.0 ** -8 + 320 * 2.0 ** -24) * np.abs(top).mean(0) + 2.0 ** -8 * np.abs(top.mean(0))
            near(out[0, :, 0], np.broadcast_to(top.mean(0), (L, d)), np.broadcast_to(tol, (L, d)), f"{exponent} {sign}")
            x = sign * d * table(fmt)[code] * 2.0 ** (exponent + (sign > 0)) / 8
            near(lse[0, :, 0], np.full(L, x + np.log(len(top))), np.full(L, 5 * 2.0 ** -24 * abs(x) + 2.0 ** -20), "lse")


@pytest.mark.parametrize("fmt,positions", [("int8", 1), ("e4m3", 1), ("int8", 700), ("e4m3", 700)])
@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_a_row_with_one_key_has_its_value(forced, form, parts, fmt, positions):
    """Where one key has all of the weight nothing is rounded but the result: half a step of it, 2^-18 for some forty steps of fp32, and 700 exp(-32)
    < 2^-36 of the others' values: a query is stretched until its best key is 32 or more ahead."""
    forced(form, parts)
    S, L, H, Hkv, d = 3, 4, 8, 4, 64
    host = Cache(S, Hkv, d, positions, 32, fmt, seed=3)
    q = torch.randn((S, L, H, d), generator=torch.Generator().manual_seed(8))
    want, best, size = np.empty((S, L, H, d)), np.empty((S, L, H)), np.empty((S, L, H))
    for s in range(S):
        keys, values = (torch.from_numpy(x) for x in host.read(s))
        for h in range(H):
            for stretch in (True, False):
                x = q[s, :, h].double() @ keys[:, h // 2].T / d ** 0.5
                top = torch.cat([x, torch.full((L, 1), -1e9)], 1).topk(2)
                ahead = top.values[:, 0] - top.values[:, 1]
                if stretch:
                    q[s, :, h] = (q[s, :, h] * (33 / ahead.float()).clamp(min=1.0)[:, None] * 1.25).to(BF).float()
            assert (ahead > 32).all()
            want[s, :, h], best[s, :, h] = values[top.indices[:, 0], h // 2].numpy(), top.values[:, 0].numpy()
            size[s, :, h] = (q[s, :, h].double().abs() @ keys[:, h // 2].abs().T / d ** 0.5).max(1).values.numpy()
    lse = torch.empty((S, L, H), device=DEV)
    out = psd.psd_attention_kv8(q.to(BF).to(DEV), host.device(DEV), lse=lse)
    near(out, want, (2.0 ** -8 + 2.0 ** -18) * np.abs(want) + 2.0 ** -36 * np.nanmax(np.abs(want)), "out")
    near(lse, best, (d + 16) * 2.0 ** -24 * size + 2.0 ** -20, "lse")


@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_zero_scales_hide_nothing(forced, form, parts):
    """A block of zeros has a scale of 0: its positions still draw weight, also in a unit's last tile."""
    forced(form, parts)
    host = Cache(1, 1, 64, 50, 16, "int8")
    host.scales[0, 0, 1:] = 0.0
    q = torch.randn((1, 2, 2, 64), generator=torch.Generator().manual_seed(1)).to(BF)
    want = attention(q, host, 1)
    out, lse = None, torch.empty((1, 2, 2), device=DEV)
    out = psd.psd_attention_kv8(q.to(DEV), host.device(DEV), lse=lse)
    near(out, want["out"], want["out_tol"], "out")
    near(lse, want["lse"], want["lse_tol"], "lse")


@pytest.mark.parametrize("form,parts", [(-1, 0), (0, 0), (1, 0), (0, 2), (1, 2)])
def test_rows_without_a_number_and_lengths_out_of_range(forced, form, parts):
    """A query of NaN spoils its own row alone, also where all that it sees has a scale of 0; lengths outside the cache are cut to it."""
    forced(form, parts)
    host = Cache(2, 1, 64, 150, 32, "e4m3", lens=[-5, 1000])
    q = torch.randn((2, 8, 8, 64), generator=torch.Generator().manual_seed(6)).to(BF)
    want = attention(q, host, 1)
    q[1, 2, 3, 10] = float("nan")
    for zero in (False, True):
        if zero:
            host.scales[:] = 0.0
        lse = torch.empty((2, 8, 8), device=DEV)
        out = psd.psd_attention_kv8(q.to(DEV), host.device(DEV), lse=lse)
        assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()
        assert torch.isnan(out[1, 2, 3]).all() and torch.isnan(lse[1, 2, 3])
        out[1, 2, 3], lse[1, 2, 3] = 0.0, 0.0
        if zero:
            assert (out == 0).all() and torch.allclose(lse[1].flatten()[lse[1].flatten() != 0], torch.tensor(float(np.log(150)), device=DEV), atol=2.0 ** -20)
        else:
            want["out"][1, 2, 3], want["lse"][1, 2, 3] = 0.0, 0.0
            near(out, want["out"], want["out_tol"], "out")
            near(lse, want["lse"], want["lse_tol"], "lse")


def test_offsets_beyond_32_bits():
    """A unit of more than 4 GB and units further apart than that: what the last head holds at both ends, and attention over its beginning."""
    Hkv, d, n = 17, 128, 1 << 20                       # 268 MB a head
    codes = torch.empty((2 * Hkv * 2 * n * d,), dtype=torch.uint8, device=DEV).view(2, Hkv, n // 32, 2, 32 * d)
    cache = psd.Kv8Cache(codes, torch.empty((2, Hkv, n // 32, 2), device=DEV), d)
    assert cache.codes.stride(0) > 2 ** 32 and Hkv * cache.codes.stride(1) > 2 ** 32
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((2, 40, Hkv, d), generator=g).to(BF) for _ in range(2))
    small = Cache(2, Hkv, d, 40, 32, "int8")
    number, scales = stored(small, k.double().numpy(), v.double().numpy(), [0, 0], [40, 40])
    for first in (n - 64, 0):
        psd.psd_kv8_store(cache, k.to(DEV), v.to(DEV), first=first)
        got = psd.psd_kv8_load(cache, first, 40, dtype=F32)
        for i in (0, 1):
            want = (number[i][:, :, :40] * scales[i][:, :, np.arange(40) // 32, None].astype(np.float64)).swapaxes(1, 2).astype(np.float32)
            assert np.array_equal(got[i].cpu().numpy(), want)
    small.codes, small.scales = codes[:, :, :2].cpu().numpy(), cache.scales[:, :, :2].cpu().numpy()
    q = torch.randn((2, 2, 2 * Hkv, d), generator=g).to(BF)
    want = attention(q, small, 1)
    out = psd.psd_attention_kv8(q.to(DEV), psd.Kv8Cache(codes, cache.scales, d, length=n, lens=torch.tensor([40, 40], dtype=torch.int32, device=DEV)))
    near(out, want["out"], want["out_tol"], "out")


@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_a_row_does_not_depend_on_what_other_sequences_hold(forced, form, parts):
    forced(form, parts)
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn((4, 3, n, 64), generator=g).to(BF).to(DEV) for n in (4, 2, 2))
    host = Cache(2, 2, 64, 200, 32, "int8")
    a = psd.psd_attention_kv8(q, host.device(DEV, per=2), k, v)
    host.codes[1] = 127
    k[3] *= 30
    b = psd.psd_attention_kv8(q, host.device(DEV, per=2), k, v)
    assert torch.equal(a[:2], b[:2]) and not torch.equal(a[2:], b[2:])


def chain(dtype, S, L, H, Hkv, d, per, fmt):
    """The way of a block: projection rows -> rotated -> attended beside the cache -> stored; twice, the second behind the first."""
    g = torch.Generator().manual_seed(S + L)
    n0, fr = 45, psd.rotary_frequencies(d // 2, 10000.0)[0].to(DEV)
    gain = torch.ones(d, device=DEV)
    units = S // per
    lens = torch.zeros(units, dtype=torch.int32, device=DEV)
    cache = psd.Kv8Cache.empty(units, Hkv, d, n0 + 2 * L, format=fmt, device=DEV, lens=lens, seqs_per_unit=per)
    prompt = torch.randn((units, n0, 2 * Hkv, d), generator=g).to(dtype).to(DEV)
    blocks = [torch.randn((S, L, H + 2 * Hkv, d), generator=g).to(dtype).to(DEV) for _ in range(2)]
    outs = [torch.empty((S, L, H, d), dtype=dtype, device=DEV) for _ in range(2)]
    ws = psd.psd_attention_kv8_workspace(outs[0], cache, blocks[0][:, :, H:H + Hkv], blocks[0][:, :, H + Hkv:])
    rotated = torch.empty_like(blocks[0][:, :, :H]), torch.empty_like(blocks[0][:, :, H:H + Hkv])
    start = torch.zeros(units, dtype=torch.int32, device=DEV)

    def go():
        lens.zero_()
        psd.psd_kv8_store(cache, prompt[:, :, :Hkv], prompt[:, :, Hkv:], first=0)
        lens.add_(n0)
        for i, b in enumerate(blocks):
            psd.psd_rotary(b[:, :, :H], b[:, :, H:H + Hkv], fr, first=n0 + i * L, q_gain=gain, k_gain=gain, q_out=rotated[0], k_out=rotated[1])
            psd.psd_attention_kv8(rotated[0], cache, rotated[1], b[:, :, H + Hkv:], out=outs[i], ws=ws)
            # the first draft of each request is kept
            start.copy_(lens)
            psd.psd_kv8_store(cache, rotated[1][::per].contiguous(), b[::per, :, H + Hkv:].contiguous(), starts=start)
            lens.add_(L)
    return go, cache, blocks, outs, rotated, lens


@pytest.mark.parametrize("dtype,S,L,H,Hkv,d,per,fmt", [(BF, 4, 32, 8, 2, 128, 2, "int8"), (BF, 3, 1, 4, 4, 64, 1, "e4m3"), (F32, 2, 16, 4, 4, 16, 1, "int8")])
def test_the_way_of_a_block_captured_and_replayed(dtype, S, L, H, Hkv, d, per, fmt):
    go, cache, blocks, outs, rotated, lens = chain(dtype, S, L, H, Hkv, d, per, fmt)
    go()
    torch.cuda.synchronize()
    eager = [o.clone() for o in outs]
    state = cache.codes.clone(), cache.scales.clone()
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        go()
    for i in range(3):
        for o in outs:
            o.fill_(float("nan"))
        cache.codes[:, :, :1].zero_()
        cache.scales[:, :, :1].fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), i
        n = (45 + 2 * L) // 32      # whole tiles that are stored
        assert torch.equal(cache.codes[:, :, :n], state[0][:, :, :n]) and torch.equal(cache.scales[:, :, :n], state[1][:, :, :n])


def test_the_way_of_a_block_against_64_bits():
    """Whole blocks of 32 behind a prompt of 64: what attention saw is what is read back afterwards."""
    S, L, H, Hkv, d, fmt = 2, 32, 4, 2, 64, "int8"
    g = torch.Generator().manual_seed(8)
    cache = psd.Kv8Cache.empty(S, Hkv, d, 128, format=fmt, device=DEV)
    freq = psd.rotary_frequencies(d, 10000.0)[0].to(DEV)
    prompt = torch.randn((S, 64, 2 * Hkv, d), generator=g).to(BF).to(DEV)
    _, k0 = psd.psd_rotary(prompt[:, :, :Hkv], prompt[:, :, :Hkv], freq)
    psd.psd_kv8_store(cache, k0, prompt[:, :, Hkv:])
    block = torch.randn((S, L, H + 2 * Hkv, d), generator=g).to(BF).to(DEV)
    q, k = psd.psd_rotary(block[:, :, :H], block[:, :, H:H + Hkv], freq, first=64)
    v = block[:, :, H + Hkv:]
    held = psd.Kv8Cache(cache.codes, cache.scales, d, length=64)
    out = psd.psd_attention_kv8(q, held, k, v)
    psd.psd_kv8_store(cache, k, v, first=64)
    host = Cache(S, Hkv, d, 64, 32, fmt)
    host.n, host.codes, host.scales = 128, cache.codes.cpu().numpy(), cache.scales.cpu().numpy()
    want = attention(q.cpu(), host, 1, k.cpu(), v.cpu())
    near(out, want["out"], want["out_tol"], "out")
    # the cache stands for the rotated keys within half a step of a whole number times the block's scale, and half a bf16 step of the value read
    back, _ = psd.psd_kv8_load(cache, 64, 32)
    scale = torch.from_numpy(host.scales[:, :, 2, 0]).to(DEV)[:, None, :, None]
    assert ((back.float() - k.float()).abs() <= scale * (0.5 + 2.0 ** -16) + 2.0 ** -8 * back.float().abs()).all()


def test_two_calls_at_once_with_a_workspace_each():
    host = Cache(2, 2, 128, 5000, 32, "int8")
    q = torch.randn((2, 1, 8, 128), generator=torch.Generator().manual_seed(2)).to(BF).to(DEV)
    cache = host.device(DEV)
    want = psd.psd_attention_kv8(q, cache)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(psd.psd_attention_kv8(q, cache))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
