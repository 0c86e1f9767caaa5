"""Model calls over keys that a batch shares: a common prefix, the sequences' own caches, weights of the cached positions, eviction.

Checked against the oracle: (1) prefix + extended caches + block rows equal its masked forward over the whole sequence, stage-1 shape
and a verification batch, fp32 within 1e-4 and bf16 within 2e-2 (the bounds of the cached calls); (2) a free-running fp32 decode
reproduces its decode token for token; (3) the weights are its attention probabilities, summed; (4) a bidirectional model under
an evicted approximate cache equals its forward over the entries that stayed.  And that the model calls, eviction and decoding run
as one program, in any order that the documentation allows."""
import dataclasses

import numpy as np
import pytest
import torch

import psd_inputs as inp
from oracle import psd_oracle as orc
from tests.shared_common import kept_positions

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _bc(shape, **kw):
    return dataclasses.replace(shape, attention="block_causal", **kw)


FP32 = inp.cut_down(inp.WORKLOADS[4].shape, name="sh-fp32", dtype="fp32", n_layers=2, d_model=96, n_heads=6, n_kv_heads=2, d_head=16, d_ffn=160,
                    vocab=211, seed=61)
BF16 = {
    "mha-dh64": inp.cut_down(inp.WORKLOADS[2].shape, n_layers=2, vocab=5000, seed=62),
    "gqa-bias-dh128": inp.cut_down(inp.WORKLOADS[4].shape, n_layers=2, d_model=512, n_heads=4, n_kv_heads=2, d_ffn=640, vocab=3001, seed=63),
}
MODELS = {"fp32": (FP32, 1e-4), **{k: (v, 2e-2) for k, v in BF16.items()}}


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _batch(shape, B, P, own, L, seed, n_committed=5, blocks_behind=1):
    """B sequences: P common tokens, `own` of their own, a block with some tokens committed, masked blocks behind."""
    N = P + own + (1 + blocks_behind) * L
    common = inp.draw_prompt(shape.vocab, P, seed) if P else np.zeros(0, dtype=np.int32)
    rng = np.random.default_rng(seed)
    rows = []
    for b in range(B):
        t = np.full(N, shape.mask_id, dtype=np.int32)
        t[:P] = common
        if own:
            t[P:P + own] = inp.draw_prompt(shape.vocab, own, seed + 10 + b)
        idx = rng.choice(L, size=n_committed + b, replace=False)
        t[P + own + idx] = rng.integers(0, shape.vocab - 1, size=n_committed + b)
        rows.append(t)
    return np.stack(rows), P + own


def _against(z, logits, top1, conf, t, mask_id, start, L, tol, label):
    """Block rows against the oracle's logits z [L, V].  With logits off by at most e everywhere, a predicted token's logit is within
    2 e of the largest, and the log of its probability within 2 e of the oracle's for that token (its own logit and the normaliser
    are off by e each) -- plus 1e-5 for a confidence that is computed in fp32 and, in bf16 models, summed from unrounded logits."""
    err = float(np.abs(logits - z).max())
    assert err <= tol, f"{label}: logits off by {err:.3e}"
    blk = t[start:start + L]
    masked = blk == mask_id
    assert (top1[~masked] == blk[~masked]).all() and (conf[~masked] == -1.0).all(), label
    y = z.copy()
    y[:, mask_id] = -np.inf
    top = y.max(-1)
    log_p = y - (top + np.log(np.exp(y - top[:, None]).sum(-1)))[:, None]
    for j in np.nonzero(masked)[0]:
        assert top1[j] != mask_id and y[j, top1[j]] >= top[j] - 2 * err - 1e-6, f"{label}: row {j}"
        assert abs(np.log(conf[j]) - log_p[j, top1[j]]) <= 2 * err + 1e-5, f"{label}: confidence of row {j}"
    return err


def _check(shape, host, logits, top1, conf, t, start, L, tol, label):
    _, _, z = orc.forward_confidence(host, t, start, L, return_logits=True, block_causal=True)
    return _against(z, logits, top1, conf, t, shape.mask_id, start, L, tol, label)


def _prefilled(psd, model, d, P, own, L, capacity):
    """SharedKv of a batch: the first sequence's prefix for all, everything behind it block by block into the caches."""
    B = d.shape[0]
    kv = psd.SharedKv(cache=psd.KvCache(model, B, capacity))
    if P:
        kv.prefix, kv.prefix_len = psd.KvCache(model, 1, P + 16), P
        psd.psd_kv_prefill(model, d[:1], P, L, kv.prefix)
    for at in range(0, own, L):
        psd.psd_kv_extend_shared(model, d, P + at, L, kv)
        kv.length += L
    return kv


@pytest.mark.parametrize("name", list(MODELS))
@pytest.mark.parametrize("L,P,own", [(16, 48, 32), (32, 96, 64), (64, 64, 0), (32, 0, 32)])
def test_shared_calls_match_the_oracle(name, L, P, own):
    import paper_2605_15609_amd as psd
    shape, tol = MODELS[name]
    shape = _bc(shape)
    B, K = 2, 3
    t, start = _batch(shape, B, P, own, L, 7)
    N = t.shape[1]
    host = inp.draw_model(shape, N)
    model = psd.Model.from_host(host, DEV)
    d = _dev(t)
    kv = _prefilled(psd, model, d, P, own, L, own + L)
    print(f"[shared model] {name} L={L} P={P} own={own}", flush=True)
    top1, conf, logits = psd.psd_forward_confidence_shared(model, d, start, L, kv, want_logits=True)
    logits = logits.cpu().numpy().reshape(B, L, -1)
    for b in range(B):
        err = _check(shape, host, logits[b], top1[b].cpu().numpy(), conf[b].cpu().numpy(), t[b], start, L, tol, f"{name} sequence {b}")
        print(f"[shared model]   sequence {b}: logits off by {err:.2e}", flush=True)
    # a verification batch: K drafts to a cache
    rng = np.random.default_rng(5)
    drafts = np.repeat(t, K, axis=0)
    for i, row in enumerate(drafts):
        masked = np.nonzero(row[start:start + L] == shape.mask_id)[0][:2 * (i % K)]
        row[start + masked] = rng.integers(0, shape.vocab - 1, size=len(masked))
    top1, conf, logits = psd.psd_forward_confidence_shared(model, _dev(drafts), start, L, kv, seqs_per_cache=K, want_logits=True)
    logits = logits.cpu().numpy().reshape(B * K, L, -1)
    for i in (1, 2, K, 2 * K - 1):
        _check(shape, host, logits[i], top1[i].cpu().numpy(), conf[i].cpu().numpy(), drafts[i], start, L, tol, f"{name} draft {i}")


@pytest.mark.parametrize("graph_kind", ["chain", "lattice"])
def test_free_running_decode_reproduces_the_oracle(graph_kind):
    import paper_2605_15609_amd as psd
    from tests.gpu_common import oracle_graph
    shape = _bc(FP32, logit_scale=6.0)
    L, P, own, B = 16, 32, 16, 3
    t, start = _batch(shape, B, P, own, L, 21, n_committed=0)
    t[:, start:] = shape.mask_id
    N = t.shape[1]
    host = inp.draw_model(shape, N)
    model = psd.Model.from_host(host, DEV)
    d = _dev(t)
    kv = _prefilled(psd, model, d, P, own, L, own + 2 * L)
    graph = psd.chain_graph(3) if graph_kind == "chain" else psd.lattice_graph(2)
    policy = psd.Policy(0.5, 1)
    stats = None
    for block in range(2):
        stats = psd.psd_decode_block_shared(model, d, start + block * L, L, policy, graph, kv, stats)
        kv.length += L
    out = d.cpu().numpy()
    for b in range(B):
        want, ostats = orc.decode(orc.model_confidence_fn(host, block_causal=True), t[b], start, L, orc.Policy(0.5, 1), oracle_graph(graph), shape.mask_id)
        assert (out[b] == want).all(), f"sequence {b}"
        assert stats[b].invocations == ostats.invocations and stats[b].tokens == ostats.tokens == 2 * L
    print(f"[shared model] decode {graph_kind}: {[s.invocations for s in stats]} invocations", flush=True)


def _record_probabilities(monkeypatch):
    """What the oracle's attention gives every key: a list of [H, Nq, Nk] arrays, one per call."""
    seen = []
    plain = orc.attention

    def attention(q, k, v, operands=None, visible=None):
        group = q.shape[1] // k.shape[1]
        p = []
        for j in range(q.shape[1]):
            s = q[:, j] @ k[:, j // group].T / np.sqrt(q.shape[2])
            if visible is not None:
                s = np.where(visible, s, -np.inf)
            e = np.exp(s - s.max(axis=-1, keepdims=True))
            p.append(e / e.sum(axis=-1, keepdims=True))
        seen.append(np.stack(p))
        return plain(q, k, v, operands, visible)
    monkeypatch.setattr(orc, "attention", attention)
    return seen


def test_weights_are_the_probabilities_of_every_layer(monkeypatch):
    import paper_2605_15609_amd as psd
    shape = _bc(FP32)
    L, P, own, B = 16, 48, 32, 2
    t, start = _batch(shape, B, P, own, L, 31)
    host = inp.draw_model(shape, t.shape[1])
    model = psd.Model.from_host(host, DEV)
    d = _dev(t)
    kv = _prefilled(psd, model, d, P, own, L, own + L)
    kv.prefix_weights, kv.cache_weights = kv.prefix.new_weights(), kv.cache.new_weights()
    psd.psd_forward_confidence_shared(model, d, start, L, kv)
    first = kv.cache_weights.clone()
    psd.psd_forward_confidence_shared(model, d, start, L, kv)
    assert torch.allclose(kv.cache_weights, 2 * first, rtol=1e-6, atol=0)      # a second call adds as much again
    H, Hkv = shape.n_heads, shape.n_kv_heads
    prefix = np.zeros((shape.n_layers, Hkv, P))
    for b in range(B):
        seen = _record_probabilities(monkeypatch)
        orc.forward_hidden(host, t[b], None, L)
        monkeypatch.undo()
        for li in range(shape.n_layers):
            w = seen[li][:, start:start + L].sum(1).reshape(Hkv, H // Hkv, -1).sum(1)      # [Hkv, positions]
            prefix[li] += w[:, :P]
            got = first[b, li].double().cpu().numpy()
            # fp32 through two layers: scores off by 1e-5 (the logits are held to 1e-4), so probabilities by that factor
            assert np.abs(got[:, :own] / w[:, P:P + own] - 1).max() < 1e-4, (b, li)
            assert (got[:, own:] == 0).all()
    got = kv.prefix_weights[0, :, :, :P].double().cpu().numpy() / 2
    assert np.abs(got / prefix - 1).max() < 1e-4
    assert (kv.prefix_weights[..., P:] == 0).all()


@pytest.mark.parametrize("name", list(MODELS))
def test_bidirectional_model_under_an_evicted_approximate_cache(name):
    import paper_2605_15609_amd as psd
    shape, tol = MODELS[name]
    L, P, G, keep, first, last = 32, 70, 64, 41, 4, 8
    N, start = P + G, P
    host = inp.draw_model(shape, N)
    model = psd.Model.from_host(host, DEV)
    t0 = np.full(N, shape.mask_id, dtype=np.int32)
    t0[:P] = inp.draw_prompt(shape.vocab, P, 41)
    t = t0.copy()
    t[start:start + 9] = inp.draw_prompt(shape.vocab, 9, 42)
    cache = psd.KvCache(model, 1, N - L)
    psd.psd_forward_confidence_approx(model, _dev(t0[None]), start, L, cache, refresh=True)
    kv = psd.SharedKv(cache=cache, length=N - L, cache_weights=cache.new_weights())
    d = _dev(t[None])
    # whole: the approximate cache's own call
    top1, conf, logits = psd.psd_forward_confidence_shared(model, d, start, L, kv, want_logits=True)
    _, _, same = psd.psd_forward_confidence_approx(model, d, start, L, cache, refresh=False, want_logits=True)
    assert float((logits - same).abs().max()) < tol
    # evicted: the oracle's forward over the entries that stayed, head by head
    small = psd.KvCache(model, 1, 48)
    weights = small.new_weights()
    kept = psd.psd_kv_evict(cache.segment(N - L, kv.cache_weights), small.segment(48, weights), keep, first, last)
    w = kv.cache_weights[0].cpu().numpy()
    kept = kept.cpu().numpy().reshape(shape.n_layers, shape.n_kv_heads, keep)
    for li in range(shape.n_layers):
        for g in range(shape.n_kv_heads):
            assert kept[li, g].tolist() == kept_positions(w[li, g], N - L, keep, first, last)
            assert np.array_equal(weights[0, li, g, :keep].cpu().numpy(), w[li, g, kept[li, g]])
    ocache = orc.ApproximateCache(host)
    ocache(t0, start, L)
    frozen = [(np.stack([k[kept[li, g], g] for g in range(shape.n_kv_heads)], 1), np.stack([v[kept[li, g], g] for g in range(shape.n_kv_heads)], 1))
              for li, (k, v) in enumerate(ocache.frozen)]
    y = orc.forward_hidden_frozen(host, t, start, L, frozen)
    z = shape.logit_scale * (y @ np.asarray(host.lm_head, dtype=np.float64).T)
    kv2 = psd.SharedKv(cache=small, length=keep)
    top1, conf, logits = psd.psd_forward_confidence_shared(model, d, start, L, kv2, want_logits=True)
    err = _against(z, logits.cpu().numpy(), top1[0].cpu().numpy(), conf[0].cpu().numpy(), t, shape.mask_id, start, L, tol, f"{name} evicted")
    print(f"[shared model] {name} evicted {N - L} -> {keep}: logits off by {err:.2e}", flush=True)


@pytest.mark.parametrize("name", list(BF16))
def test_a_served_batch_under_a_budget(name):
    """A common prompt, four requests behind it, decoded block by block; after every block the requests' caches are cut to a budget by
    what their positions drew.  Equal to the same requests decoded one at a time on the fp32-exact parts (positions, lengths),
    every token resolved, the prefix untouched."""
    import paper_2605_15609_amd as psd
    shape = _bc(BF16[name])
    L, P, own, B, blocks, keep = 32, 96, 32, 4, 3, 40
    t, start = _batch(shape, B, P, own, L, 51, n_committed=0, blocks_behind=blocks - 1)
    model = psd.Model.from_host(inp.draw_model(shape, t.shape[1]), DEV)
    d = _dev(t)
    kv = _prefilled(psd, model, d, P, own, L, keep + L)
    before = kv.prefix.mem.clone()
    other = psd.KvCache(model, B, keep + L)
    kv.cache_weights = kv.cache.new_weights()
    other_weights = other.new_weights()
    for block in range(blocks):
        psd.psd_decode_block_shared(model, d, start + block * L, L, psd.Policy(0.9, 4), psd.chain_graph(3), kv)
        kv.length += L
        assert (kv.cache_weights[..., :kv.length - L] > 0).all() and (kv.cache_weights[..., kv.length:] == 0).all()
        if kv.length > keep:
            other_weights.zero_()
            kept = psd.psd_kv_evict(kv.cache.segment(kv.length, kv.cache_weights), other.segment(keep + L, other_weights), keep, 4, L)
            kept = kept.cpu().numpy()
            assert (np.diff(kept, axis=-1) > 0).all() and (kept[..., :4] == np.arange(4)).all() and (kept[..., -L:] == np.arange(kv.length - L, kv.length)).all()
            kv.cache, other = other, kv.cache
            kv.cache_weights, other_weights = other_weights, kv.cache_weights
            kv.length = keep
    assert not (d == shape.mask_id).any()
    assert torch.equal(kv.prefix.mem, before)


def test_shared_calls_refuse():
    import paper_2605_15609_amd as psd
    shape = _bc(BF16["mha-dh64"])
    L = 32
    model = psd.Model.from_host(inp.draw_model(shape, 256), DEV)
    bid = psd.Model.from_host(inp.draw_model(BF16["mha-dh64"], 256), DEV)
    d = torch.zeros((2, 256), dtype=torch.int32, device=DEV)
    cache, prefix = psd.KvCache(model, 2, 64), psd.KvCache(model, 1, 64)
    ok = dict(prefix=prefix, prefix_len=64, cache=cache, length=32)

    def kv(**kw):
        return psd.SharedKv(**dict(ok, **kw))
    psd.psd_forward_confidence_shared(model, d, 96, L, kv())
    psd.psd_forward_confidence_shared(model, d, 96, L, kv(length=64))
    for bad in (kv(prefix_len=65), kv(prefix_len=-1), kv(length=65), kv(length=-1), kv(prefix=None), kv(cache=None), kv(cache=psd.KvCache(model, 1, 64)),
                kv(cache_weights=prefix.new_weights()), kv(prefix_weights=prefix.new_weights().double()), kv(prefix=psd.KvCache(bid, 1, 64))):
        with pytest.raises(psd.PsdError):
            psd.psd_forward_confidence_shared(model, d, 96, L, bad)
    for start, length in ((96, 24), (240, 32), (-1, 32), (96, 0)):
        with pytest.raises(psd.PsdError):
            psd.psd_forward_confidence_shared(model, d, start, length, kv())
    with pytest.raises(psd.PsdError):
        psd.psd_forward_confidence_shared(model, d, 96, L, kv(), seqs_per_cache=3)
    with pytest.raises(psd.PsdError):
        psd.psd_kv_extend_shared(model, d, 96, L, kv(length=33))
    with pytest.raises(psd.PsdError):
        psd.psd_decode_block_shared(model, d, 96, L, psd.Policy(), psd.chain_graph(2), kv(length=33))
    with pytest.raises(psd.PsdError):
        psd.psd_kv_extend_shared(bid, d, 96, L, psd.SharedKv(cache=psd.KvCache(bid, 2, 64), length=0))
    small = torch.empty(4096, dtype=torch.uint8, device=DEV)
    import ctypes as C
    c = kv().c(model, 2)
    top1, conf = torch.empty((2, L), dtype=torch.int32, device=DEV), torch.empty((2, L), device=DEV)
    assert model.lib.psd_forward_confidence_shared(model.handle, d.data_ptr(), 2, 256, 96, L, C.byref(c), top1.data_ptr(), conf.data_ptr(), None,
                                                   small.data_ptr(), 4096, None) == -3


@pytest.mark.parametrize("L,P,own,K", [(16, 96, 16, 3), (32, 96, 96, 4)])
def test_one_request_whose_drafts_share_a_tile(L, P, own, K):
    """Few heads: the rows of all drafts are one tile, which walks prefix, cache and every draft's block, cut into more parts than the
    segments have steps of 32 keys."""
    import paper_2605_15609_amd as psd
    shape, tol = MODELS["gqa-bias-dh128"]
    shape = _bc(shape)
    t, start = _batch(shape, 1, P, own, L, 71)
    N = t.shape[1]
    host = inp.draw_model(shape, N)
    model = psd.Model.from_host(host, DEV)
    kv = _prefilled(psd, model, _dev(t), P, own, L, own + L)
    rng = np.random.default_rng(6)
    drafts = np.repeat(t, K, axis=0)
    for i, row in enumerate(drafts):
        masked = np.nonzero(row[start:start + L] == shape.mask_id)[0][:2 * i]
        row[start + masked] = rng.integers(0, shape.vocab - 1, size=len(masked))
    print(f"[shared model] one tile L={L} P={P} own={own} K={K}", flush=True)
    top1, conf, logits = psd.psd_forward_confidence_shared(model, _dev(drafts), start, L, kv, seqs_per_cache=K, want_logits=True)
    logits = logits.cpu().numpy().reshape(K, L, -1)
    for i in range(K):
        _check(shape, host, logits[i], top1[i].cpu().numpy(), conf[i].cpu().numpy(), drafts[i], start, L, tol, f"draft {i}")
    d = _dev(t)
    psd.psd_decode_block_shared(model, d, start, L, psd.Policy(0.9, 1), psd.chain_graph(K), kv)
    assert not (d[:, start:start + L] == shape.mask_id).any()


def test_shared_calls_refuse_memory_that_they_would_add_to_twice():
    import paper_2605_15609_amd as psd
    shape = _bc(BF16["mha-dh64"])
    L = 32
    model = psd.Model.from_host(inp.draw_model(shape, 256), DEV)
    d = torch.zeros((2, 256), dtype=torch.int32, device=DEV)
    cache, prefix = psd.KvCache(model, 2, 96), psd.KvCache(model, 1, 64)
    rows = (shape.n_layers, shape.n_kv_heads)
    n_prefix, n_cache = rows[0] * rows[1] * 64, 2 * rows[0] * rows[1] * 96
    buf = torch.zeros((n_prefix + n_cache,), device=DEV)

    def kv(at_prefix, at_cache, **kw):
        return psd.SharedKv(**dict(dict(prefix=prefix, prefix_len=64, cache=cache, length=32, prefix_weights=buf[at_prefix:at_prefix + n_prefix].view(1, *rows, 64),
                                        cache_weights=buf[at_cache:at_cache + n_cache].view(2, *rows, 96)), **kw))
    decode = (psd.Policy(), psd.chain_graph(2))
    psd.psd_forward_confidence_shared(model, d, 96, L, kv(0, n_prefix))
    psd.psd_forward_confidence_shared(model, d, 96, L, kv(n_cache, 0))
    psd.psd_forward_confidence_shared(model, d, 96, L, kv(0, 0, length=0))       # (nothing cached, nothing to add to)
    for bad in (kv(0, 0), kv(0, n_prefix - 1), kv(n_cache - 1, 0)):
        with pytest.raises(psd.PsdError, match="same weights"):
            psd.psd_forward_confidence_shared(model, d, 96, L, bad)
        with pytest.raises(psd.PsdError, match="same weights"):
            psd.psd_decode_block_shared(model, d, 96, L, *decode, bad)
    on_keys = prefix.mem[:n_prefix * 4].view(torch.float32).view(1, *rows, 64)
    with pytest.raises(psd.PsdError, match="weights lie on"):
        psd.psd_forward_confidence_shared(model, d, 96, L, kv(0, n_prefix, prefix_weights=on_keys))
    one = psd.KvCache(model, 1, 96)
    for length in (0, 32, 64):
        both = psd.SharedKv(prefix=one, prefix_len=64, cache=one, length=length)
        with pytest.raises(psd.PsdError, match="the prefix is one of"):
            psd.psd_kv_extend_shared(model, d[:1], 96, L, both)
        with pytest.raises(psd.PsdError, match="the prefix is one of"):
            psd.psd_decode_block_shared(model, d[:1], 96, L, *decode, both)
    psd.psd_forward_confidence_shared(model, d[:1], 96, L, psd.SharedKv(prefix=one, prefix_len=64, cache=one, length=32))   # (read only)


def _block_behind(host, t, start, L, frozen):
    """Oracle: logits of the block rows behind `frozen` ((keys, values) of every layer), and the rows' own (keys, values)."""
    cos, sin = np.asarray(host.rope_cos[start:start + L], dtype=np.float64), np.asarray(host.rope_sin[start:start + L], dtype=np.float64)
    h, own = np.asarray(host.tok_emb, dtype=np.float64)[t[start:start + L]], []
    for lw, kv in zip(host.layers, frozen):
        h = orc.layer_forward(h, lw, host.shape, cos, sin, None, None, own, kv)
    y = orc.rmsnorm(h, np.asarray(host.final_norm, dtype=np.float64), host.shape.rms_eps)
    return host.shape.logit_scale * (y @ np.asarray(host.lm_head, dtype=np.float64).T), own


def _evicted(shape, seed, L, P, own, keep, first, last):
    """Two requests whose caches of `own` positions were cut to `keep`: (psd, host, model, tokens, start, SharedKv, oracle's entries of each)."""
    import paper_2605_15609_amd as psd
    B = 2
    t, start = _batch(shape, B, P, own, L, seed, blocks_behind=1)
    host = inp.draw_model(shape, t.shape[1])
    model = psd.Model.from_host(host, DEV)
    kv = _prefilled(psd, model, _dev(t), P, own, L, own + L)
    kv.cache_weights = kv.cache.new_weights()
    psd.psd_forward_confidence_shared(model, _dev(t), start, L, kv)
    small = psd.KvCache(model, B, keep + 2 * L)
    kept = psd.psd_kv_evict(kv.cache.segment(own, kv.cache_weights), small.segment(keep + 2 * L), keep, first, last)
    kept = kept.cpu().numpy().reshape(B, shape.n_layers, shape.n_kv_heads, keep)
    frozen = []
    for b in range(B):
        seen = []
        orc.forward_hidden(host, t[b], None, L, seen)
        frozen.append([tuple(np.concatenate([x[:P], np.stack([x[P + kept[b, li, g], g] for g in range(shape.n_kv_heads)], 1)]) for x in kv_)
                       for li, kv_ in enumerate(seen)])
    return psd, host, model, t, start, psd.SharedKv(prefix=kv.prefix, prefix_len=P, cache=small, length=keep), frozen


@pytest.mark.parametrize("name", list(MODELS))
@pytest.mark.parametrize("L,keep", [(16, 41), (32, 40), (16, 63)])
def test_a_block_goes_behind_a_length_that_is_no_multiple_of_16(name, L, keep):
    """Eviction leaves any length.  The block behind it, its keys and values in the cache, and the block after that, against the oracle's
    forward over the entries that stayed."""
    from tests.shared_common import slots
    shape, tol = MODELS[name]
    shape = _bc(shape)
    psd, host, model, t, start, kv, frozen = _evicted(shape, 81, L, 48 if L == 16 else 64, 64, keep, 4, 8)
    B, w = 2, shape.n_kv_heads * shape.d_head
    print(f"[shared model] {name} L={L} behind {keep}", flush=True)

    def block(at, behind):
        top1, conf, logits = psd.psd_forward_confidence_shared(model, _dev(t), at, L, kv, want_logits=True)
        logits, rows = logits.cpu().numpy().reshape(B, L, -1), []
        for b in range(B):
            z, own = _block_behind(host, t[b], at, L, behind[b])
            _against(z, logits[b], top1[b].cpu().numpy(), conf[b].cpu().numpy(), t[b], shape.mask_id, at, L, tol, f"{name} sequence {b} at {at}")
            rows.append(own)
        return rows
    block(start, frozen)
    t[:, start:start + L] = np.stack([inp.draw_prompt(shape.vocab, L, 90 + b) for b in range(B)])
    before = kv.cache.segment(keep + 2 * L)
    k_before, vt_before = before.k.clone(), before.vt.clone()
    psd.psd_kv_extend_shared(model, _dev(t), start, L, kv)
    kv.length += L
    rows = block(start + L, [[(np.concatenate([k, r[0]]), np.concatenate([v, r[1]])) for (k, v), r in zip(frozen[b], _block_behind(host, t[b], start, L, frozen[b])[1])]
                             for b in range(B)])
    # what was written, and what was not
    after = kv.cache.segment(keep + 2 * L)
    k, vt = after.k.float().cpu().numpy(), after.vt.float().cpu().numpy()
    at = np.arange(keep, keep + L)
    slot = slots(keep + L).numpy()[at]
    other = np.ones(vt.shape[2], dtype=bool)
    other[slot] = False
    assert torch.equal(after.k[:, :keep], k_before[:, :keep]) and torch.equal(after.k[:, keep + L:], k_before[:, keep + L:])
    assert torch.equal(after.vt[:, :, torch.from_numpy(other)], vt_before[:, :, torch.from_numpy(other)])
    # The first layer's, element by element: the norm's output, the projection and its rotation are rounded to the model's type (u each, two
    # channels meet in a rotation), sums of d_model products are fp32
    u, d = (0.0 if shape.dtype == "fp32" else 2.0 ** -8), shape.d_model
    rel = u + (d + 16) * 2.0 ** -24
    for b in range(B):
        a = orc.rmsnorm(np.asarray(host.tok_emb, dtype=np.float64)[t[b, start:start + L]], np.asarray(host.layers[0]["attn_norm"], dtype=np.float64), shape.rms_eps)
        want = _block_behind(host, t[b], start, L, frozen[b])[1][0]
        size_k, size_v = (np.abs(a) @ np.abs(np.asarray(host.layers[0][m], dtype=np.float64)).T for m in ("wk", "wv"))
        if host.layers[0].get("bk") is not None:
            size_k, size_v = size_k + np.abs(host.layers[0]["bk"]), size_v + np.abs(host.layers[0]["bv"])
        size_k = size_k.reshape(L, shape.n_kv_heads, 2, shape.d_head // 2).sum(2)      # (the two channels of a rotation are half a head apart)
        size_k = np.concatenate([size_k, size_k], -1).reshape(L, w)
        got_k, got_v = k[b * shape.n_layers, at], vt[b * shape.n_layers][:, slot].T
        assert (np.abs(got_k - want[0].reshape(L, w)) <= 3.1 * rel * size_k).all() and (np.abs(got_v - want[1].reshape(L, w)) <= 2.1 * rel * size_v).all(), b


@pytest.mark.parametrize("graph_kind", ["chain", "lattice"])
def test_requests_decoded_together_behind_evicted_caches(graph_kind):
    """fp32, two blocks each: together, one at a time, and the oracle's decode over the entries that stayed give the same tokens."""
    from tests.gpu_common import oracle_graph
    shape, L = _bc(FP32, logit_scale=6.0), 16
    psd, host, model, t, start, kv, frozen = _evicted(shape, 82, L, 32, 64, 37, 4, 16)
    t[:, start:] = shape.mask_id
    graph = psd.chain_graph(3) if graph_kind == "chain" else psd.lattice_graph(2)
    policy, oracle_policy = psd.Policy(0.5, 1), orc.Policy(0.5, 1)
    singles, per_seq = [], kv.cache.segment(37).k.shape[0] // 2
    for b in range(2):
        one = psd.KvCache(model, 1, kv.cache.capacity)
        a, c = kv.cache.segment(37), one.segment(37)
        c.k.copy_(a.k[b * per_seq:(b + 1) * per_seq])
        c.vt.copy_(a.vt[b * per_seq:(b + 1) * per_seq])
        singles.append(psd.SharedKv(prefix=kv.prefix, prefix_len=kv.prefix_len, cache=one, length=37))
    together, alone = _dev(t), [_dev(t[b:b + 1]) for b in range(2)]
    want = [t[b].copy() for b in range(2)]
    for n in range(2):
        at = start + n * L
        psd.psd_decode_block_shared(model, together, at, L, policy, graph, kv)
        kv.length += L
        for b in range(2):
            psd.psd_decode_block_shared(model, alone[b], at, L, policy, graph, singles[b])
            singles[b].length += L
            entries = frozen[b]

            def confidence(tokens, block_start, length):
                z, _ = _block_behind(host, np.asarray(tokens), block_start, length, entries)
                x, c = orc.top1_confidence(z, shape.mask_id)
                blk = np.asarray(tokens)[block_start:block_start + length]
                return np.where(blk == shape.mask_id, x, blk).astype(np.int32), np.where(blk == shape.mask_id, c, -1.0).astype(np.float32)
            want[b], _ = orc.decode_block(confidence, want[b], at, L, oracle_policy, oracle_graph(graph), shape.mask_id)
            own = _block_behind(host, want[b], at, L, entries)[1]
            frozen[b] = [(np.concatenate([k, r[0]]), np.concatenate([v, r[1]])) for (k, v), r in zip(entries, own)]
    for b in range(2):
        got = together[b].cpu().numpy()
        assert (got == alone[b][0].cpu().numpy()).all() and (got == want[b]).all(), b
