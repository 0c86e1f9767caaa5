"""Operators whose speed is measured: attention over keys that a batch shares, the attention weights that its keys
collect, and the eviction of cached positions by those weights.

  attend  psd_attention_shared: S sequences of L rows attend to segments of keys, coarse to fine -- a prefix that the
          whole batch shares, a cache for every `drafts` consecutive sequences (the drafts of one request), and, where
          the drafts differ, the rows of the block itself
  weigh   the same with the softmax's log-sum kept, then psd_attention_weights: what every cached key has drawn
  evict   psd_kv_evict: of every cache, layer and KV head the `keep` positions that drew most (the first and the last
          ones always), keys, values and weights gathered into another cache

Keys are rows of n_kv_heads * d_head channels; values are transposed, [n_kv_heads * d_head, positions], the positions of
every group of 16 in the order 0-3, 8-11, 4-7, 12-15 (the caches of this package).  Shapes: the heads, blocks and drafts
of this repository's configurations.
"""
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
#: query heads, KV heads, width of a head
HEADS = {"8B": (32, 32, 128), "7B": (28, 4, 128), "small": (8, 8, 64), "tiny": (4, 4, 16)}


def _attend(name, op, heads, S, L, prefix, cache, drafts=1, block=False, ragged=False, dtype="bf16"):
    c = {"op": op, "heads": heads, "S": S, "L": L, "prefix": prefix, "cache": cache, "drafts": drafts, "block": block, "ragged": ragged,
         "dtype": dtype}
    return dict(c, name=name) if name else c


def _evict(name, heads, seqs, layers, length, keep, first, last, ragged=False, dtype="bf16"):
    c = {"op": "evict", "heads": heads, "seqs": seqs, "layers": layers, "length": length, "keep": keep, "first": first, "last": last,
         "ragged": ragged, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # four users of a small model behind a short common instruction, one row each: launches and latency
        _attend("small, single rows", "attend", "small", 4, 1, 256, 61, ragged=True),
        # the fp32 type at a size of its tests, blocks of 16, lengths of no round number
        _attend("small fp32, blocks", "attend", "small", 3, 16, 333, 77, ragged=True, dtype="fp32"),
        # one row each of 32 requests on one document, grouped KV heads: the document's keys are read once or 32 times
        _attend("7B, single rows, long document", "attend", "7B", 32, 1, 32768, 300, ragged=True),
        # blocks of 16 requests behind one instruction, MHA: stage 1 of a batch
        _attend("8B, blocks", "attend", "8B", 16, 32, 1024, 288, ragged=True),
        # six drafts of four requests: shared instruction, the request's cache, the draft's own block
        _attend("7B, drafts", "attend", "7B", 24, 32, 2077, 519, drafts=6, block=True),
        # the verification of a full batch, 128 drafts of 64 rows, behind a long shared prompt
        _attend("8B, batch of 128 drafts", "attend", "8B", 128, 64, 4096, 1024, drafts=8, block=True),
        # weights that one block of a user gives the 480 frozen positions around it (approximate cache, third configuration)
        _attend("8B weights, one block", "weigh", "8B", 1, 32, 0, 480, block=True),
        # weights over a shared document and the caches of 16 requests
        _attend("7B weights, batch", "weigh", "7B", 16, 64, 2048, 4001, ragged=True),
        # the same in fp32 at the smallest heads there are
        _attend("tiny fp32 weights", "weigh", "tiny", 2, 16, 100, 45, ragged=True, dtype="fp32"),
        # one user of the small model: 352 positions around a block down to 128
        _evict("small eviction", "small", 1, 8, 352, 128, 4, 16),
        # a long prompt of an 8B model down to a quarter, all layers
        _evict("8B eviction", "8B", 1, 32, 4096, 1024, 4, 32),
        # caches of five requests of unequal length, grouped KV heads, some of them within the budget already
        _evict("7B ragged eviction", "7B", 5, 28, 2003, 500, 0, 64, ragged=True),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def spread(lo, hi):      # whole numbers, evenly over their logarithm
        return int(round(lo * (hi / lo) ** rng.random()))

    most = max(_cost(c) for c in listed())
    while True:
        dtype = "fp32" if rng.random() < 0.25 else "bf16"
        heads = rng.choice(["small", "tiny"] if dtype == "fp32" else ["small", "7B", "8B"])
        op = rng.choice(["attend", "attend", "attend", "weigh", "weigh", "evict", "evict"])
        if op == "evict":
            length = spread(17, 16384)
            keep = spread(max(1, length // 16), length)
            case = _evict("", heads, spread(1, 8), spread(1, 32), length, keep, rng.choice([0, 4, keep // 4]), rng.choice([0, 16, keep // 2]),
                          rng.random() < 0.4, dtype)
            _, Hkv, dh = HEADS[heads]
            # (the caches themselves stay within 12 GB)
            if case["first"] + case["last"] > keep or case["seqs"] * case["layers"] * length * Hkv * dh > 3e9 / (1 if dtype == "bf16" else 2):
                continue
        else:
            drafts, block = rng.choice([(1, False), (1, True), (rng.randint(2, 8), True)])
            prefix, cache = rng.choice([0, spread(16, 32768), spread(16, 32768)]), rng.choice([0, spread(1, 8192), spread(1, 1024)])
            if dtype == "fp32":
                prefix, cache = prefix // 16, cache // 8
            L = rng.choice([1, 1, 16, 32, 48, 64, rng.randint(2, 63)])
            case = _attend("", op, heads, drafts * spread(1, 32), L, prefix, cache, drafts, block, rng.random() < 0.5, dtype)
            if prefix + cache < 1:
                continue
        if _cost(case) <= most:
            return case


# --------------------------------------------------------------------------------------------------------------- inputs
def _slots(n, device=DEVICE):
    """Where position 0 .. n-1 stands in a transposed value row."""
    j = torch.arange(n, device=device)
    piece = (j >> 2) & 3
    return (j & ~15) | ((((piece & 1) << 1) | (piece >> 1)) << 2) | (j & 3)


def _segments(case):
    """(name, units, sequences to a unit, positions) of the segments that a case has, coarse to fine."""
    S, n = case["S"], case["drafts"]
    all_of_them = [("prefix", 1, S, case["prefix"]), ("cache", S // n, n, case["cache"]), ("block", S, 1, case["L"] if case["block"] else 0)]
    return [s for s in all_of_them if s[3]]


def _prepare_attention(case, g):
    H, Hkv, dh = HEADS[case["heads"]]
    dtype, S, L = DTYPES[case["dtype"]], case["S"], case["L"]

    def normal(*dims):
        return torch.empty(dims, dtype=dtype, device=DEVICE).normal_(generator=g)

    # every KV head has a direction that its queries lean to and that a few of the keys have much of: some positions draw
    # most of the weight, as in trained models
    lean = normal(Hkv, 1, dh)
    q = 1.5 * normal(S, L, Hkv, H // Hkv, dh) + 0.5 * lean
    state = {"case": case, "q": q.view(S, L, H, dh), "segments": []}
    for name, units, per_unit, n in _segments(case):
        k = normal(units, n, Hkv, dh)
        k += 0.1 * torch.empty((units, n, Hkv, 1), dtype=dtype, device=DEVICE).normal_(generator=g).square() * lean.view(Hkv, dh)
        lens = None
        if case["ragged"] and name == "cache":      # a request's own part may be as short as one position
            lens = torch.randint(1, n + 1, (units,), generator=g, device=DEVICE, dtype=torch.int32)
        weighed = case["op"] == "weigh" and name != "block"
        state["segments"].append({
            "k": k.view(units, n, Hkv * dh), "vt": normal(units, Hkv * dh, (n + 63) // 64 * 64), "lens": lens, "per_unit": per_unit,
            "weights": torch.zeros((units, Hkv, n), dtype=torch.float32, device=DEVICE) if weighed else None})
    state["out"] = torch.empty((S, L, H, dh), dtype=dtype, device=DEVICE)
    state["lse"] = torch.empty((S, L, H), dtype=torch.float32, device=DEVICE) if case["op"] == "weigh" else None
    if own:
        import paper_2605_15609_amd as psd
        state["psd"] = psd
        state["keys"] = psd.KvSegments([psd.KvSegment(s["k"], s["vt"], dh, seqs_per_unit=s["per_unit"], lens=s["lens"], weights=s["weights"])
                                        for s in state["segments"]])
        state["ws"] = psd.psd_attention_workspace(state["q"], state["keys"])
    return state


def _prepare_evict(case, g):
    _, Hkv, dh = HEADS[case["heads"]]
    dtype, n, keep, units = DTYPES[case["dtype"]], case["length"], case["keep"], case["seqs"] * case["layers"]

    def cache(capacity, fill):
        k = torch.zeros((units, capacity, Hkv * dh), dtype=dtype, device=DEVICE)
        vt = torch.zeros((units, Hkv * dh, (capacity + 63) // 64 * 64), dtype=dtype, device=DEVICE)
        w = torch.zeros((units, Hkv, capacity), dtype=torch.float32, device=DEVICE)
        if fill:
            k.normal_(generator=g)
            vt.normal_(generator=g)
            # a few positions drew most of the weight, many next to nothing, some nothing at all
            w.uniform_(generator=g).pow_(4)
            w[w < 1e-3] = 0.0
        return {"k": k, "vt": vt, "weights": w}

    lens = None
    if case["ragged"]:      # every layer of a request holds as much
        lens = torch.randint(1, n + 1, (case["seqs"],), generator=g, device=DEVICE, dtype=torch.int32).repeat_interleave(case["layers"])
    state = {"case": case, "src": cache(n, True), "dst": cache(keep, False), "lens": lens,
             "kept": torch.empty((units, Hkv, keep), dtype=torch.int32, device=DEVICE),
             "kept_lens": torch.empty((units,), dtype=torch.int32, device=DEVICE)}
    if own:
        import paper_2605_15609_amd as psd
        state["psd"] = psd
        s, d = state["src"], state["dst"]
        state["from"] = psd.KvSegment(s["k"], s["vt"], dh, lens=lens, weights=s["weights"])
        state["to"] = psd.KvSegment(d["k"], d["vt"], dh, weights=d["weights"])
    return state


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return _prepare_evict(case, g) if case["op"] == "evict" else _prepare_attention(case, g)


# ----------------------------------------------------------------------------------------------------- one pass, plain form
def _scores(q, s):
    """Scores of every row against its unit's keys, [S, Hkv, L * group, n] in 32 bits, -inf where a unit holds fewer."""
    S, L, H, dh = q.shape
    units, n, width = s["k"].shape
    Hkv = width // dh
    rows = q.float().view(units, S // units * L, Hkv, H // Hkv, dh).permute(0, 2, 1, 3, 4).reshape(units, Hkv, -1, dh)
    x = torch.matmul(rows, s["k"].float().view(units, n, Hkv, dh).permute(0, 2, 3, 1).contiguous()) / dh ** 0.5
    if s["lens"] is not None:
        x = x.masked_fill((torch.arange(n, device=x.device) >= s["lens"][:, None])[:, None, None, :], float("-inf"))
    return x.view(units, Hkv, S // units, -1, n).transpose(1, 2).reshape(S, Hkv, -1, n)


def _part(p, s, S, dh):
    """sum_j p_j v_j over a segment, [S, Hkv, L * group, dh]."""
    units, width, _ = s["vt"].shape
    Hkv, n = width // dh, s["k"].shape[1]
    v = s["vt"].float()[:, :, _slots(n)].view(units, Hkv, dh, n).transpose(2, 3).contiguous()
    if s["lens"] is not None:
        v = v * (torch.arange(n, device=v.device) < s["lens"][:, None])[:, None, :, None]
    rows = p.reshape(units, S // units, Hkv, -1, n).transpose(1, 2).reshape(units, Hkv, -1, n)
    return torch.matmul(rows, v).view(units, Hkv, S // units, -1, dh).transpose(1, 2).reshape(S, Hkv, -1, dh)


def _attention(state):
    q, segments = state["q"], state["segments"]
    S, L, H, dh = q.shape
    x = torch.cat([_scores(q, s) for s in segments], dim=-1)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(torch.where(top.isinf(), torch.zeros_like(top), top)))
    total = p.sum(-1, keepdim=True)
    parts = p.div_(torch.where(total > 0, total, torch.ones_like(total))).split([s["k"].shape[1] for s in segments], dim=-1)
    out = sum(_part(w, s, S, dh) for w, s in zip(parts, segments))
    Hkv = out.shape[1]

    def by_head(t):
        return t.view(S, Hkv, L, H // Hkv, -1).permute(0, 2, 1, 3, 4).reshape(S, L, H, -1)

    answer = {"out": by_head(out).to(q.dtype)}
    if state["lse"] is not None:
        answer["lse"] = by_head(top + total.log())[..., 0]
        answer["weights"] = [w.sum(2).view(s["k"].shape[0], -1, Hkv, w.shape[-1]).sum(1) if s["weights"] is not None else None
                             for w, s in zip(parts, segments)]
    return answer


def _eviction(state):
    case, src, dst = state["case"], state["src"], state["dst"]
    units, Hkv, n = src["weights"].shape
    keep, dh = case["keep"], src["k"].shape[2] // Hkv
    lens = state["lens"] if state["lens"] is not None else torch.full((units,), n, dtype=torch.int32, device=DEVICE)
    j, end = torch.arange(n, device=DEVICE), lens[:, None, None]
    w = src["weights"].masked_fill((j < case["first"]) | (j >= end - case["last"]), float("inf")).masked_fill(j >= end, float("-inf"))
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    kept = order.masked_fill(order >= end, n).sort(-1).values                      # ascending; n where a cache holds fewer
    there, at = kept < n, kept.clamp(max=n - 1)
    k = src["k"].view(units, n, Hkv, dh).gather(1, at.transpose(1, 2)[..., None].expand(-1, -1, -1, dh))
    k = torch.where(there.transpose(1, 2)[..., None], k, dst["k"].view(units, keep, Hkv, dh))
    ld = dst["vt"].shape[-1]
    v = src["vt"].view(units, Hkv, dh, -1).gather(3, _slots(n)[at][:, :, None, :].expand(-1, -1, dh, -1))
    vt = dst["vt"].view(units, Hkv, dh, ld).clone()
    vt[..., _slots(keep)] = torch.where(there[:, :, None, :], v, vt[..., _slots(keep)])
    return {"k": k.reshape(units, keep, -1), "vt": vt.view(units, -1, ld), "kept": kept.masked_fill(~there, -1).int(),
            "lens": lens.clamp(max=keep).int(), "weights": torch.where(there, src["weights"].gather(2, at), dst["weights"])}


# ------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if not own:
        return _eviction(state) if case["op"] == "evict" else _attention(state)
    psd = state["psd"]
    if case["op"] == "evict":
        psd.psd_kv_evict(state["from"], state["to"], case["keep"], first=case["first"], last=case["last"], kept=state["kept"],
                         kept_lens=state["kept_lens"])
        d = state["dst"]
        return {"k": d["k"], "vt": d["vt"], "kept": state["kept"], "lens": state["kept_lens"], "weights": d["weights"]}
    psd.psd_attention_shared(state["q"], state["keys"], out=state["out"], lse=state["lse"], ws=state["ws"])
    if case["op"] == "attend":
        return {"out": state["out"]}
    psd.psd_attention_weights(state["q"], state["keys"], state["lse"], accumulate=False)
    return {"out": state["out"], "lse": state["lse"], "weights": [s["weights"] for s in state["segments"]]}


# ------------------------------------------------------------------------------------------------- what a pass cannot avoid
def work(case):
    H, Hkv, dh = HEADS[case["heads"]]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "evict":
        units = case["seqs"] * case["layers"]
        # lengths of a ragged batch are even over 1 .. length
        n, keep = case["length"], case["keep"]
        held, kept = ((n + 1) / 2, keep - keep * (keep - 1) / (2.0 * n)) if case["ragged"] else (n, keep)
        return {"bytes": units * Hkv * (4.0 * held + kept * (2 * 2 * dh * size + 8)), "flops": float(units * Hkv * held)}
    rows, nbytes, flops = case["S"] * case["L"] * H, 0.0, 0.0
    for name, units, per_unit, n in _segments(case):
        held = (n + 1) / 2 if case["ragged"] and name == "cache" else n
        nbytes += units * held * Hkv * 2 * dh * size
        flops += 4.0 * rows * dh * held
        if case["op"] == "weigh" and name != "block":
            nbytes += 4.0 * units * Hkv * held
            flops += rows * held
    return {"bytes": nbytes + rows * (2 * dh * size + (4 if case["op"] == "weigh" else 0)), "flops": flops}


def _cost(case):
    # in seconds; the plain forms hold every score, so those count as well
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] * (1 if case["dtype"] == "bf16" else 10) / 1e15


# ------------------------------------------------------------------------------------------------------- what is right
def _exact_attention(case, state):
    """Request by request (all sequences of one cache), every row against the list of the positions that it sees."""
    q, segments = state["q"], state["segments"]
    S, L, H, dh = q.shape
    Hkv = HEADS[case["heads"]][1]
    out = torch.zeros((S, L, H, dh), dtype=torch.float64, device=q.device)
    lse = torch.zeros((S, L, H), dtype=torch.float64, device=q.device)
    weights = [None if s["weights"] is None else torch.zeros(s["weights"].shape, dtype=torch.float64, device=q.device) for s in segments]
    for s in range(S):
        keys, values, where = [], [], []
        for i, seg in enumerate(segments):
            u = s // seg["per_unit"]
            n = seg["k"].shape[1] if seg["lens"] is None else int(seg["lens"][u])
            keys.append(seg["k"][u, :n].double())
            values.append(seg["vt"][u].double().t()[_slots(n)])
            where.append((i, u, n))
        k, v = torch.cat(keys).view(-1, Hkv, dh), torch.cat(values).view(-1, Hkv, dh)
        for g in range(Hkv):
            at = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
            rows = q[s, :, at].double().reshape(-1, dh)
            x = rows.mm(k[:, g].t().contiguous()) / float(dh) ** 0.5
            z = x.logsumexp(-1)
            p = (x - z[:, None]).exp()
            out[s, :, at] = p.mm(v[:, g].contiguous()).view(L, -1, dh)
            lse[s, :, at] = z.view(L, -1)
            begin = 0
            for i, u, n in where:
                if weights[i] is not None:
                    weights[i][u, g, :n] += p[:, begin:begin + n].sum(0)
                begin += n
    return {"out": out} if case["op"] == "attend" else {"out": out, "lse": lse, "weights": weights}


def _exact_eviction(case, state):
    """Cache by cache: everything over the smallest weight that stays, and of those equal to it the first ones."""
    src, dst, keep = state["src"], state["dst"], case["keep"]
    units, Hkv, n = src["weights"].shape
    dh = src["k"].shape[2] // Hkv
    answer = {"k": dst["k"].double(), "vt": dst["vt"].double(), "kept": torch.full((units, Hkv, keep), -1, dtype=torch.int32, device=DEVICE),
              "lens": torch.zeros((units,), dtype=torch.int32, device=DEVICE), "weights": dst["weights"].double()}
    for u in range(units):
        held = n if state["lens"] is None else int(state["lens"][u])
        m = min(held, keep)
        w = src["weights"][u, :, :held].double()
        w[:, :case["first"]] = float("inf")
        w[:, max(0, held - case["last"]):] = float("inf")
        least = w.topk(m, dim=-1).values[:, -1:]
        over, equal = w > least, w == least
        stays = over | (equal & (equal.cumsum(-1) <= m - over.sum(-1, keepdim=True)))
        at = stays.nonzero()[:, 1].view(Hkv, m)
        heads = torch.arange(Hkv, device=DEVICE)[:, None]
        answer["k"][u, :m] = src["k"][u].view(n, Hkv, dh)[at, heads].transpose(0, 1).reshape(m, -1).double()
        values = src["vt"][u].view(Hkv, dh, -1).transpose(1, 2)[heads, _slots(n)[at]]
        answer["vt"][u].view(Hkv, dh, -1)[:, :, _slots(m)] = values.transpose(1, 2).double()
        answer["kept"][u, :, :m] = at.int()
        answer["lens"][u] = m
        answer["weights"][u, :, :m] = src["weights"][u].double()[heads, at]
    return answer


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_eviction(case, state) if case["op"] == "evict" else _exact_attention(case, state)
