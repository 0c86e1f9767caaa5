"""8-bit caches and rotation on the GPU where numbers, lengths and forms end."""
import numpy as np
import pytest
import torch

import paper_2605_15609_amd as psd
from paper_2605_15609_amd import binding as B
from tests.gpu_common import DEV
from tests.kv8_common import Cache, spots, stored, table
from tests.shared_common import near
from tests.test_gpu_kv8 import check_store, forced, run_attention  # noqa: F401 (forced: a fixture)

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

#: largest magnitudes of a block, in units of the smallest number: quotients by a scale of so few bits pass the largest code by up to half of it
TINY = [1, 2, 63, 64, 65, 127, 150, 190, 191, 223, 224, 225, 337, 449, 465, 500, 671, 672, 1119, 1121, 5000, 6047, 8953, 9999, 16385, 123457, 2 ** 19 - 1, 2 ** 19,
        2 ** 21 + 1, 2 ** 22 + 3, 2 ** 23 - 1, 2 ** 23 + 5]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [16, 64, 128])
def test_blocks_of_the_smallest_numbers(fmt, d):
    """fp32 rows whose scales are below the normal numbers, in fresh blocks and behind kept rows: codes and scales are exact, and what is read back is
    code * scale (a whole number of smallest ones in int8; rounded to one in e4m3)."""
    units, rng = len(TINY), np.random.default_rng(d)
    host = Cache(units, 1, d, 32, 32, fmt, seed=d)
    dev = host.device(DEV)

    def rows(tops):
        x = np.stack([rng.integers(-t, t + 1, (16, 1, d)) for t in tops]).astype(np.float64)
        for u, t in enumerate(tops):
            x[u, 5, 0, 7], x[u, 6, 0, 9] = t, -t
        return torch.from_numpy(x * 2.0 ** -149).to(F32)
    for start, tops in ((0, TINY), (16, TINY[::-1])):
        k, v = rows(tops), rows(tops[1:] + tops[:1])
        number, scales = stored(host, k.double().numpy(), v.double().numpy(), [start] * units, [16] * units)
        check_store(host, dev, k, v, [start] * units, [16] * units, call=dict(first=start))
        host.codes, host.scales = dev.codes.cpu().numpy(), dev.scales.cpu().numpy()
        for got, n, s in zip(psd.psd_kv8_load(dev, 0, start + 16, dtype=F32), number, scales):
            want = (n[:, :, :start + 16] * s.astype(np.float64)[..., None]).swapaxes(1, 2).astype(np.float32)
            assert np.isfinite(want).all() and np.array_equal(got.cpu().numpy(), want)


def test_products_below_the_normal_numbers_are_rounded_once():
    """e4m3 codes times scales of 2^-149 whole numbers, next to a border between two numbers of bf16 by less than fp32 has there."""
    t = table("e4m3")
    host, pairs = Cache(1, 1, 16, 64 * 16, 16, "e4m3"), []
    for byte in (0x0b, 0x14, 0x1d, 0x25, 0x2b, 0x33, 0x35, 0x37):
        for m in range(12):
            # code * k 2^-149 beside (2 m + 1) 2^-134, by half of 2^-149 at most
            k = round((2 * m + 1) * 2 ** 15 / t[byte])
            if 0 < k < 2 ** 23 and k * t[byte] != (2 * m + 1) * 2 ** 15:
                pairs.append((byte, k))
    pairs = pairs[:64]
    assert len(pairs) == 64
    flat = host.codes.reshape(1, 1, -1)
    for b, (byte, k) in enumerate(pairs):
        for at in spots(host.n, 16):
            flat[0, 0, at[16 * b:16 * b + 16]] = byte
            flat[0, 0, at[16 * b + 3]] = byte | 0x80
        host.scales[0, 0, b] = np.float32(k * 2.0 ** -149)
    want = host.read(0)[0]
    # exact, and rounded to whole numbers of 2^-133, ties to even
    want = np.sign(want) * np.rint(np.abs(want) * 2.0 ** 133) * 2.0 ** -133
    assert (want != 0).any()
    for got in psd.psd_kv8_load(host.device(DEV), 0, 16 * len(pairs)):
        assert np.array_equal(got[0].double().cpu().numpy(), want[:16 * len(pairs)])


@pytest.mark.parametrize("none", [0.0, 2.0 ** -130, 2.0 ** -149])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("L,positions", [(4, 200), (64, 200), (64, 700)])
@pytest.mark.parametrize("form,parts", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_a_row_with_one_key_beside_blocks_without_values(forced, form, parts, fmt, L, positions, none):
    """Blocks whose values are all zero (a scale of 0), or too small for a reciprocal of their scale: a row that a key of another block has all of is still
    rounded once -- half a step, 2^-18 for some forty steps of fp32, and 700 exp(-32) < 2^-36 of the others' values."""
    forced(form, parts)
    d = 64
    host = Cache(1, 1, d, positions, 16, fmt, seed=11)
    without = np.arange(host.n // 16) % 2 == 1                  # every second block, so every step of every wavefront has one
    host.scales[0, 0, without & ~np.isnan(host.scales[0, 0, :, 1]), 1] = none
    host.scales[0, 0, ~np.isnan(host.scales[0, 0, :, 0]), 0] = 0.02
    keys, values = (torch.from_numpy(x[:, 0]) for x in host.read(0))
    # each row asks for a key of its own, of a block that has values
    held = torch.from_numpy(np.flatnonzero(~without[np.arange(positions) // 16]))
    best = held[torch.arange(2 * L) * 37 % len(held)]
    q = (keys[best] * (1000 / (keys[best] ** 2).sum(1, keepdim=True))).to(BF)
    top = (q.double() @ keys.T / d ** 0.5).topk(2)
    assert torch.equal(top.indices[:, 0], best) and (top.values[:, 0] - top.values[:, 1] > 33).all()
    want = values[best].view(1, L, 2, d).numpy()
    out = psd.psd_attention_kv8(q.view(1, L, 2, d).to(DEV), host.device(DEV))
    near(out, want, (2.0 ** -8 + 2.0 ** -18) * np.abs(want) + 2.0 ** -36 * np.abs(values.numpy()).max(), "out")


def parts_of(form, positions, parts):
    """Parts that a call of so many positions has when `parts` are asked for: whole steps of 128 (form 0) or 64 positions, evenly."""
    steps = max(1, -(-positions // (64 if form else 128)))
    each = -(-steps // min(parts, steps))
    return -(-steps // each)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("parts", [1, 2, 3, 5])
@pytest.mark.parametrize("dtype,form,H,Hkv,d,S,L,per,positions,lens,own", [
    (BF, 0, 28, 4, 128, 2, 1, 1, 1000, [1000, 129], True), (BF, 1, 8, 2, 64, 4, 33, 2, 700, [700, 65], True), (BF, 1, 4, 1, 128, 2, 64, 2, 449, None, False),
    (F32, 0, 4, 4, 16, 2, 5, 1, 600, [600, 1], True), (F32, 0, 2, 1, 128, 2, 64, 1, 900, None, True), (F32, 0, 8, 8, 64, 4, 3, 2, 385, [385, 0], False)])
def test_as_many_parts_as_were_asked_for(forced, fmt, parts, dtype, form, H, Hkv, d, S, L, per, positions, lens, own):
    forced(form, parts)
    plan = run_attention(dtype, H, Hkv, d, S, L, per, positions, 32, fmt, lens, own, seed=positions + parts)
    assert (plan[0], plan[2]) == (form, parts_of(form, positions, parts)) and (parts == 1) == (plan[2] == 1)


@pytest.mark.parametrize("form,parts", [(0, 1), (1, 1), (0, 2), (1, 2)])
def test_every_position_of_a_cache_of_zeros_counts(forced, form, parts):
    """All scales are 0: every score is 0, so lse is the log of the number of positions in every row."""
    forced(form, parts)
    host = Cache(2, 1, 64, 150, 32, "e4m3", lens=[33, 150])
    host.scales[:] = 0.0
    q = torch.randn((2, 8, 8, 64), generator=torch.Generator().manual_seed(6)).to(BF).to(DEV)
    lse = torch.full((2, 8, 8), float("nan"), device=DEV)
    out = psd.psd_attention_kv8(q, host.device(DEV), lse=lse)
    assert (out == 0).all()
    near(lse, np.log(np.array([33.0, 150.0]))[:, None, None] * np.ones((1, 8, 8)), np.full((2, 8, 8), 2.0 ** -20), "lse")


def test_two_calls_at_once_that_both_need_a_workspace():
    host = Cache(2, 2, 128, 5000, 32, "int8")
    q = torch.randn((2, 1, 8, 128), generator=torch.Generator().manual_seed(2)).to(BF).to(DEV)
    cache = host.device(DEV)
    assert B.attention_kv8_plan(q, cache)[2] > 1
    spaces = [psd.psd_attention_kv8_workspace(q, cache) for _ in range(2)]
    assert spaces[0].numel() > 256
    others = q.flip(0).contiguous()
    want = [psd.psd_attention_kv8(x, cache) for x in (q, others)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.full_like(q, float("nan")) for _ in range(12)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        with torch.cuda.stream(streams[i % 2]):
            psd.psd_attention_kv8((q, others)[i % 2], cache, out=out, ws=spaces[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i % 2]) for i, o in enumerate(outs))
