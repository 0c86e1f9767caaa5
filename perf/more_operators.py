"""Operators whose speed is measured: the way of a block's rows into a cache of 8-bit codes and the attention that reads it.

  rotate  psd_rotary: queries and keys of every head normed (or not) and rotated by their positions, in halves or neighbouring
          pairs, the whole head or its first channels, frequencies as they are or scaled for long contexts
  store   psd_kv8_store, then psd_kv8_load: keys and values of new positions into a cache that holds them in 8 bits with one scale
          for every block of positions and KV head, and what the blocks that changed stand for now
  attend  psd_attention_kv8: S sequences of L rows attend to such a cache (one for every `drafts` consecutive sequences), then to
          the rows of their own block, which are not in it

A cache is codes uint8 [units, n_kv_heads, positions / 32, 2, 32 * d_head] and scales float32 [units, n_kv_heads, positions / block,
2], keys before values in both.  Of 32 positions keys lie as [d_head / 16][32 positions][16 channels], values as [d_head / w][2][w
channels][16 positions], w = min(32, d_head), where part h of the two holds positions 8 b + 4 h + j in the order of (b, j), b and j
0 .. 3.  A code is a whole number -127 .. 127 (int8) or a float of 4 and 3 bits (e4m3); what it stands for is code * scale.  A
block's scale is its largest magnitude over the largest code, rounded to 32 bits; a block that is stored in parts keeps the largest
scale that one of them needed, and what it held before is rounded again when that grows.  Shapes: the heads, blocks and drafts of
this repository's configurations.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
#: query heads, KV heads, width of a head
HEADS = {"8B": (32, 32, 128), "7B": (28, 4, 128), "small": (8, 8, 64), "tiny": (4, 4, 16)}
#: the largest code
MOST = {"int8": 127.0, "e4m3": 448.0}
THETA = 500000.0
EPS = 1e-6


def _rotate(name, heads, S, L, first=0, part=1, interleaved=False, norm=False, stretch=1.0, dtype="bf16"):
    c = {"op": "rotate", "heads": heads, "S": S, "L": L, "first": first, "part": part, "interleaved": interleaved, "norm": norm,
         "stretch": stretch, "dtype": dtype}
    return dict(c, name=name) if name else c


def _store(name, heads, units, n, first, ragged=False, block=32, format="int8", dtype="bf16"):
    c = {"op": "store", "heads": heads, "units": units, "n": n, "first": first, "ragged": ragged, "block": block, "format": format,
         "dtype": dtype}
    return dict(c, name=name) if name else c


def _attend(name, heads, S, L, length, drafts=1, own_rows=True, ragged=False, lse=False, block=32, format="int8", dtype="bf16"):
    c = {"op": "attend", "heads": heads, "S": S, "L": L, "length": length, "drafts": drafts, "own_rows": own_rows, "ragged": ragged,
         "lse": lse, "block": block, "format": format, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the block of one user of the small model: a launch and its latency
        _rotate("small, one block", "small", 1, 32, first=256),
        # the stage-1 call of a batch of 16, heads normed before they are rotated
        _rotate("8B, batch of sequences", "8B", 16, 1280, norm=True),
        # rows of six drafts far into a long document: neighbouring pairs of the first half of a head, scaled frequencies
        _rotate("7B, part of the head", "7B", 6, 1021, first=131072, part=2, interleaved=True, stretch=8.0),
        # one token each of 32 requests, behind caches that end anywhere inside a block
        _store("7B, single tokens", "7B", 32, 1, 480, ragged=True),
        # four whole prompts of an MHA model
        _store("8B, prompts", "8B", 4, 1024, 0, format="e4m3"),
        # blocks of the fp32 type behind caches of unequal length, few positions to a scale
        _store("small fp32, stored blocks", "small", 3, 48, 333, ragged=True, block=16, dtype="fp32"),
        # one row each of four users of the small model: launches and latency
        _attend("small, single rows", "small", 4, 1, 300, ragged=True),
        # the fp32 type, blocks of 16, lengths of no round number
        _attend("small fp32, blocks", "small", 3, 16, 410, ragged=True, lse=True, block=64, dtype="fp32"),
        # one row each of 32 requests with long caches of unequal length, grouped KV heads
        _attend("7B, single rows, long caches", "7B", 32, 1, 16384, ragged=True),
        # blocks of 16 requests, MHA: stage 1 of a batch
        _attend("8B, blocks", "8B", 16, 32, 1312),
        # six drafts of four requests: the request's cache, the draft's own block
        _attend("7B, drafts", "7B", 24, 32, 2596, drafts=6, lse=True, format="e4m3"),
        # the verification of a full batch, 128 drafts of 64 rows
        _attend("8B, batch of 128 drafts", "8B", 128, 64, 5120, drafts=8),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def spread(lo, hi):      # whole numbers, evenly over their logarithm
        return int(round(lo * (hi / lo) ** rng.random()))

    most = max(_cost(c) for c in listed())
    while True:
        dtype = "fp32" if rng.random() < 0.25 else "bf16"
        heads = rng.choice(["small", "tiny"] if dtype == "fp32" else ["small", "7B", "8B"])
        H, Hkv, dh = HEADS[heads]
        op = rng.choice(["rotate", "store", "attend", "attend"])
        format, block = rng.choice(["int8", "e4m3"]), rng.choice([16, 32, 32, 64, 128])
        L = rng.choice([1, 1, 16, 32, 48, 64, rng.randint(2, 63)])
        if op == "rotate":
            rows = rng.choice([L, L, spread(65, 4096)])
            case = _rotate("", heads, spread(1, 64), rows, rng.choice([0, spread(1, 1000000)]), rng.choice([1, 1, 2, 4]), rng.random() < 0.5,
                           rng.random() < 0.5, rng.choice([1.0, 4.0, 32.0]), dtype)
            if case["S"] * rows * (H + Hkv) * dh > 3e8:
                continue
        elif op == "store":
            n = rng.choice([L, L, spread(65, 8192)])
            case = _store("", heads, spread(1, 64), n, rng.choice([0, spread(1, 8192)]), rng.random() < 0.5, block, format, dtype)
            if case["units"] * (n + 64) * Hkv * dh > 1e8:
                continue
        else:
            drafts = rng.choice([1, 1, rng.randint(2, 8)])
            length = spread(1, 4096 if dtype == "fp32" else 65536)
            case = _attend("", heads, drafts * spread(1, 64), L, length, drafts, rng.random() < 0.7, rng.random() < 0.5, rng.random() < 0.4,
                           block, format, dtype)
            # (the caches themselves stay within 1.5 GB)
            if case["S"] // drafts * length * Hkv * dh > 0.75e9:
                continue
        if _cost(case) <= most:
            return case


# --------------------------------------------------------------------------------------------------------------- inputs
def _normal(g, dtype, *dims):
    return torch.empty(dims, dtype=dtype, device=DEVICE).normal_(generator=g)


def _frequencies(rotated, stretch):
    """Radians a position of every pair, in 64 bits, and the factor on the rotated channels: as they are, or scaled part by part, the slow
    ones (less than one turn over 8192 positions) stretched, the fast ones (more than 32 turns) not, a ramp between."""
    f = THETA ** (-torch.arange(0, rotated, 2, dtype=torch.float64) / rotated)
    if stretch == 1.0:
        return f, 1.0
    fast = ((8192 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * (fast + (1.0 - fast) / stretch), 0.1 * math.log(stretch) + 1.0


def _prepare_rotate(case, g):
    H, Hkv, dh = HEADS[case["heads"]]
    dtype, S, L = DTYPES[case["dtype"]], case["S"], case["L"]
    # the rows of a QKV projection: queries and keys are columns of it
    qkv = _normal(g, dtype, S, L, H + 2 * Hkv, dh)
    freq, factor = _frequencies(dh // case["part"], case["stretch"])
    # sequences stand at positions of their own
    start = case["first"] + torch.randint(0, 1000, (S, 1), generator=g, device=DEVICE, dtype=torch.int32)
    state = {"case": case, "q": qkv[:, :, :H], "k": qkv[:, :, H:H + Hkv], "positions": start + torch.arange(L, device=DEVICE, dtype=torch.int32),
             "frequencies": freq.to(DEVICE), "factor": factor,
             "q_out": torch.empty((S, L, H, dh), dtype=dtype, device=DEVICE), "k_out": torch.empty((S, L, Hkv, dh), dtype=dtype, device=DEVICE)}
    for name in ("q_gain", "k_gain"):
        state[name] = 1.0 + 0.1 * _normal(g, torch.float32, dh) if case["norm"] else None
    return state


def _e4m3(x):
    """The nearest float of 4 and 3 bits (ties to even), up to 448, for x in 64 bits."""
    step = torch.exp2(torch.frexp(x)[1].clamp(min=-5).double() - 4)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _codes(x, format):
    return torch.round(x).clamp(-127.0, 127.0) if format == "int8" else _e4m3(x)


def _pack(keys, values, format):
    """Codes (as numbers) of keys and values [units, positions, heads, d] as a cache holds them."""
    units, n, Hkv, d = keys.shape
    tiles, w = n // 32, min(32, d)
    kind = torch.int8 if format == "int8" else torch.float8_e4m3fn
    k = keys.to(kind).view(torch.uint8).view(units, tiles, 32, Hkv, d // 16, 16).permute(0, 3, 1, 4, 2, 5)
    v = values.to(kind).view(torch.uint8).view(units, tiles, 4, 2, 4, Hkv, d // w, w).permute(0, 5, 1, 6, 3, 7, 2, 4)
    return torch.stack([k.reshape(units, Hkv, tiles, 32 * d), v.reshape(units, Hkv, tiles, 32 * d)], 3)


def _unpack(codes, d, format, which, dtype):
    """Codes of keys (0) or values (1) as numbers [units, positions, heads, d]."""
    units, Hkv, tiles = codes.shape[:3]
    w = min(32, d)
    c = codes[:, :, :, which].view(torch.int8 if format == "int8" else torch.float8_e4m3fn).to(dtype)
    if which == 0:
        return c.view(units, Hkv, tiles, d // 16, 32, 16).permute(0, 2, 4, 1, 3, 5).reshape(units, tiles * 32, Hkv, d)
    return c.view(units, Hkv, tiles, d // w, 2, w, 4, 4).permute(0, 2, 6, 4, 7, 1, 3, 5).reshape(units, tiles * 32, Hkv, d)


def _cache(case, g, units, n):
    """A cache of n positions (rounded up to whole blocks and tiles) of keys and values as a model has them: some channels are larger."""
    _, Hkv, d = HEADS[case["heads"]]
    block, format = case["block"], case["format"]
    n = -(-n // max(32, block)) * max(32, block)
    codes = torch.empty((units, Hkv, n // 32, 2, 32 * d), dtype=torch.uint8, device=DEVICE)
    scales = torch.empty((units, Hkv, n // block, 2), dtype=torch.float32, device=DEVICE)
    large = 1.0 + 2.0 * _normal(g, torch.float32, Hkv, d).abs().pow(3)
    step = max(1, int(2e8 // (n * Hkv * d)))
    for at in range(0, units, step):
        m = min(step, units - at)
        parts = []
        for i, channel in enumerate((large / large.square().mean().sqrt(), 1.0)):
            x = _normal(g, torch.float32, m, n // block, block, Hkv, d) * channel
            s = x.abs().amax((2, 4)) / MOST[format]
            scales[at:at + m, :, :, i] = s.transpose(1, 2)
            parts.append(_codes(x.div_(s[:, :, None, :, None]), format).view(m, n, Hkv, d))
        codes[at:at + m] = _pack(*parts, format)
    return codes, scales


def _prepare_store(case, g):
    _, Hkv, d = HEADS[case["heads"]]
    units, n, first, dtype = case["units"], case["n"], case["first"], DTYPES[case["dtype"]]
    starts = torch.full((units,), first, dtype=torch.int32, device=DEVICE)
    if case["ragged"]:
        starts += torch.randint(0, 64, (units,), generator=g, device=DEVICE, dtype=torch.int32)
    codes, scales = _cache(case, g, units, first + n + 63 * case["ragged"])
    large = 1.0 + 2.0 * _normal(g, dtype, Hkv, d).abs().pow(3)
    # what comes back: from the first block that may change to the last position that may be stored
    begin = first // case["block"] * case["block"]
    rows = first + n + 63 * case["ragged"] - begin
    state = {"case": case, "codes": codes, "scales": scales, "starts": starts, "lens": starts + n, "begin": begin, "rows": rows,
             "k": _normal(g, dtype, units, n, Hkv, d) * large, "v": _normal(g, dtype, units, n, Hkv, d)}
    if own:
        import paper_2605_15609_amd as psd
        state["cache"] = psd.Kv8Cache(codes, scales, d, format=case["format"], lens=state["lens"])
        for name in ("k_out", "v_out"):      # (positions behind a unit's last are left as they are)
            state[name] = torch.zeros((units, rows, Hkv, d), dtype=dtype, device=DEVICE)
    return state


def _prepare_attend(case, g):
    H, Hkv, d = HEADS[case["heads"]]
    dtype, S, L, n = DTYPES[case["dtype"]], case["S"], case["L"], case["length"]
    units = S // case["drafts"]
    codes, scales = _cache(case, g, units, n)
    lens = None
    if case["ragged"]:      # a request may be as young as one position
        lens = torch.randint(1, n + 1, (units,), generator=g, device=DEVICE, dtype=torch.int32)
    state = {"case": case, "codes": codes, "scales": scales, "lens": lens, "q": 1.5 * _normal(g, dtype, S, L, H, d),
             "k": None, "v": None, "out": torch.empty((S, L, H, d), dtype=dtype, device=DEVICE),
             "lse": torch.empty((S, L, H), dtype=torch.float32, device=DEVICE) if case["lse"] else None}
    if case["own_rows"]:      # columns of the rows that the projection leaves
        kv = _normal(g, dtype, S, L, 2 * Hkv, d)
        state["k"], state["v"] = kv[:, :, :Hkv], kv[:, :, Hkv:]
    if own:
        import paper_2605_15609_amd as psd
        state["cache"] = psd.Kv8Cache(codes, scales, d, format=case["format"], length=n, lens=lens, seqs_per_unit=case["drafts"])
        state["ws"] = psd.psd_attention_kv8_workspace(state["q"], state["cache"], state["k"], state["v"])
    return state


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return {"rotate": _prepare_rotate, "store": _prepare_store, "attend": _prepare_attend}[case["op"]](case, g)


# ----------------------------------------------------------------------------------------------------- one pass, plain form
def _rotation(state):
    case = state["case"]
    # far positions: the angle in 64 bits, its cosine and sine in 32
    angle = state["positions"].double()[:, :, None, None] * state["frequencies"]
    cos, sin = (angle.cos() * state["factor"]).float(), (angle.sin() * state["factor"]).float()
    answer = {}
    for name in ("q", "k"):
        x = state[name].float()
        if state[name + "_gain"] is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * state[name + "_gain"]
        n = 2 * cos.shape[-1]
        a, b = (x[..., 0:n:2], x[..., 1:n:2]) if case["interleaved"] else (x[..., :n // 2], x[..., n // 2:n])
        a, b = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
        answer[name] = torch.cat([turned, x[..., n:]], -1).to(state[name].dtype)
    return answer


def _storing(state):
    case, starts = state["case"], state["starts"].long()
    _, Hkv, d = HEADS[case["heads"]]
    units, n, block, format = case["units"], case["n"], case["block"], case["format"]
    capacity = state["scales"].shape[2] * block
    begin, rows = state["begin"], state["rows"]
    position = torch.arange(begin, capacity, device=DEVICE)
    row = position - starts[:, None]                                                # [units, positions]
    new, kept = (row >= 0) & (row < n), row < 0
    answer = {}
    for i, name in enumerate(("k", "v")):
        had = state["scales"][:, :, begin // block:, i].transpose(1, 2)             # [units, blocks, heads]
        # a block that begins with a new position starts afresh
        had = torch.where((position[::block] < starts[:, None])[:, :, None], had, torch.zeros_like(had))
        x = state[name].gather(1, row.clamp(0, n - 1)[:, :, None, None].expand(-1, -1, Hkv, d)).float()
        x = torch.where(new[:, :, None, None], x, torch.zeros_like(x))
        needed = (x.view(units, -1, block, Hkv, d).abs().amax((2, 4)).double() / MOST[format]).float()
        s = torch.maximum(had, needed)
        per_row = [t.double().repeat_interleave(block, 1)[..., None] for t in (had, s)]
        old = _unpack(state["codes"], d, format, i, torch.float32)[:, begin:].double() * per_row[0]
        # quotients next to a border between two codes: in 64 bits
        x = torch.where(new[:, :, None, None], x.double(), old) / torch.where(per_row[1] > 0, per_row[1], torch.ones_like(per_row[1]))
        value = (_codes(x, format) * per_row[1]).to(state[name].dtype)
        answer[name] = torch.where((new | kept)[:, :, None, None], value, torch.zeros_like(value))[:, :rows]
    return answer


def _attention(state):
    case, q = state["case"], state["q"]
    S, L, H, d = q.shape
    Hkv, drafts = HEADS[case["heads"]][1], case["drafts"]
    units, n = S // drafts, case["length"]

    def read(i):      # [units, heads, positions, d] in 32 bits
        c = _unpack(state["codes"], d, case["format"], i, torch.float32)[:, :n].transpose(1, 2)
        return (c * state["scales"][..., i].repeat_interleave(case["block"], 2)[:, :, :n, None]).contiguous()

    rows = q.float().view(units, drafts * L, Hkv, H // Hkv, d).transpose(1, 2).reshape(units, Hkv, -1, d)
    x = torch.matmul(rows, read(0).transpose(2, 3).contiguous()) / d ** 0.5
    if state["lens"] is not None:
        x = x.masked_fill((torch.arange(n, device=x.device) >= state["lens"][:, None])[:, None, None, :], float("-inf"))
    top = x.amax(-1, keepdim=True)
    if state["k"] is not None:
        mine = q.float().view(S, L, Hkv, H // Hkv, d).transpose(1, 2).reshape(S, Hkv, -1, d)
        y = torch.matmul(mine, state["k"].float().permute(0, 2, 3, 1).contiguous()) / d ** 0.5      # [S, heads, rows, L]

        def by_unit(t):
            return t.view(units, drafts, Hkv, -1, t.shape[-1]).transpose(1, 2).reshape(units, Hkv, -1, t.shape[-1])
        y = by_unit(y)
        top = torch.maximum(top, y.amax(-1, keepdim=True))
    p = torch.exp(x.sub_(top))
    total = p.sum(-1, keepdim=True)
    values = read(1)
    if state["lens"] is not None:
        values = values * (torch.arange(n, device=x.device) < state["lens"][:, None])[:, None, :, None]
    out = torch.matmul(p, values)
    if state["k"] is not None:
        e = torch.exp(y - top)
        total = total + e.sum(-1, keepdim=True)
        e = e.view(units, Hkv, drafts, -1, L).transpose(1, 2).reshape(S, Hkv, -1, L)
        out = out + by_unit(torch.matmul(e, state["v"].float().transpose(1, 2).contiguous()))

    def by_head(t):
        return t.view(units, Hkv, drafts * L, H // Hkv, -1).transpose(1, 2).reshape(S, L, H, -1)
    answer = {"out": by_head(out / total).to(q.dtype)}
    if case["lse"]:
        answer["lse"] = by_head(top + total.log())[..., 0]
    return answer


# ------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if not own:
        return {"rotate": _rotation, "store": _storing, "attend": _attention}[case["op"]](state)
    import paper_2605_15609_amd as psd
    if case["op"] == "rotate":
        psd.psd_rotary(state["q"], state["k"], state["frequencies"], positions=state["positions"], interleaved=case["interleaved"],
                       factor=state["factor"], q_gain=state["q_gain"], k_gain=state["k_gain"], eps=EPS, q_out=state["q_out"], k_out=state["k_out"])
        return {"q": state["q_out"], "k": state["k_out"]}
    if case["op"] == "store":
        psd.psd_kv8_store(state["cache"], state["k"], state["v"], starts=state["starts"])
        psd.psd_kv8_load(state["cache"], state["begin"], state["rows"], k_out=state["k_out"], v_out=state["v_out"])
        return {"k": state["k_out"], "v": state["v_out"]}
    psd.psd_attention_kv8(state["q"], state["cache"], state["k"], state["v"], out=state["out"], lse=state["lse"], ws=state["ws"])
    return {"out": state["out"], "lse": state["lse"]} if case["lse"] else {"out": state["out"]}


# ------------------------------------------------------------------------------------------------- what a pass cannot avoid
def work(case):
    H, Hkv, d = HEADS[case["heads"]]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rotate":
        channels = case["S"] * case["L"] * (H + Hkv) * d
        return {"bytes": channels * 2 * size + case["S"] * case["L"] * 4, "flops": (3.0 / case["part"] + 4.0 * case["norm"]) * channels}
    if case["op"] == "store":
        stored = case["units"] * case["n"] * Hkv * d * 2
        # of the blocks that change: what they held before, and what comes back
        before = case["first"] % case["block"] + 31.5 * case["ragged"]
        back = stored + case["units"] * before * Hkv * d * 2
        return {"bytes": stored * (size + 1.0) + back * (1.0 + size) + 8.0 * back / (2 * d * case["block"]), "flops": 3.0 * stored + back}
    rows, units = case["S"] * case["L"] * H, case["S"] // case["drafts"]
    # lengths of a ragged batch are even over 1 .. length
    held = (case["length"] + 1) / 2 if case["ragged"] else case["length"]
    mine = case["L"] if case["own_rows"] else 0
    nbytes = units * held * Hkv * (2 * d + 8.0 / case["block"]) + rows * (2 * d * size + 4 * case["lse"]) + case["S"] * mine * Hkv * 2 * d * size
    return {"bytes": nbytes, "flops": 4.0 * rows * d * (held + mine)}


def _cost(case):
    # in seconds; the plain forms hold every score and cache in 32 bits, so those count as well
    w = work(case)
    return w["bytes"] / 1e12 + w["flops"] * (1 if case["dtype"] == "bf16" else 10) / 1e15


# ------------------------------------------------------------------------------------------------------- what is right
def _exact_rotation(case, state):
    """Pair by pair as a product of complex numbers."""
    answer = {}
    n = 2 * state["frequencies"].shape[0]
    turn = torch.polar(torch.full((), float(state["factor"]), dtype=torch.float64, device=DEVICE),
                       state["positions"].double()[..., None] * state["frequencies"])[:, :, None, :]
    for name in ("q", "k"):
        x = state[name].double()
        if case["norm"]:
            x = x / ((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * state[name + "_gain"].double()
        at = torch.arange(n, device=DEVICE).view(-1, 2) if case["interleaved"] else torch.arange(n, device=DEVICE).view(2, -1).t()
        z = torch.complex(x[..., at[:, 0]], x[..., at[:, 1]]) * turn
        x[..., at[:, 0]], x[..., at[:, 1]] = z.real, z.imag
        answer[name] = x
    return answer


def _values(format):
    """What every byte stands for."""
    if format == "int8":
        return torch.tensor([b - 256 if b > 127 else b for b in range(256)], dtype=torch.float64, device=DEVICE)
    out = []
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        out.append((-1) ** (b >> 7) * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)) if b & 127 != 127 else float("nan"))
    return torch.tensor(out, dtype=torch.float64, device=DEVICE)


def _at(case, position):
    """Byte of channel 0 .. d - 1 at positions [n] among those of one KV head: keys [n, d], values [n, d]."""
    d = HEADS[case["heads"]][2]
    w = min(32, d)
    tile, r, c = position[:, None] // 32, position[:, None] % 32, torch.arange(d, device=DEVICE)
    keys = tile * 64 * d + c // 16 * 512 + r * 16 + c % 16
    values = tile * 64 * d + 32 * d + c // w * (32 * w) + r // 4 % 2 * (16 * w) + c % w * 16 + r // 8 * 4 + r % 4
    return keys, values


def _exact_store(case, state):
    """Block by block, the nearest code picked from the list of all of them."""
    _, Hkv, d = HEADS[case["heads"]]
    units, n, block, begin, rows = case["units"], case["n"], case["block"], state["begin"], state["rows"]
    table = _values(case["format"])
    kinds = table[table.abs() <= MOST[case["format"]]].unique()
    between = (kinds[1:] + kinds[:-1]) / 2
    even = torch.arange(kinds.numel(), device=DEVICE)
    middle = int((kinds == 0).nonzero())
    even = (even - middle) % 2 == 0                      # the codes on either side of 0 are odd, the next ones even, and so on
    answer = {name: torch.zeros((units, rows, Hkv, d), dtype=torch.float64, device=DEVICE) for name in ("k", "v")}
    for u in range(units):
        start = int(state["starts"][u])
        for b in range(begin // block, (start + n - 1) // block + 1):
            lo, hi = b * block, min((b + 1) * block, start + n)
            at = _at(case, torch.arange(lo, hi, device=DEVICE))
            for i, name in enumerate(("k", "v")):
                kept = min(max(start - lo, 0), hi - lo)
                had = state["scales"][u, :, b, i].double() if kept else torch.zeros(Hkv, dtype=torch.float64, device=DEVICE)
                held = table[state["codes"][u].reshape(Hkv, -1)[:, at[i][:kept]].long()].transpose(0, 1) * had[:, None]
                x = torch.cat([held, state[name][u, max(lo - start, 0):hi - start].double()]) if hi > start else held
                s = torch.maximum(had, (x[kept:].abs().amax((0, 2)) / MOST[case["format"]]).float().double()) if hi > start else had
                y = x / s.where(s > 0, torch.ones_like(s))[:, None]
                i_lo = torch.bucketize(y.contiguous(), between)       # (a quotient on a border: below it)
                tie = (i_lo < between.numel()) & (y == between[i_lo.clamp(max=between.numel() - 1)]) & ~even[i_lo]
                answer[name][u, lo - begin:hi - begin] = kinds[i_lo + tie.long()] * s[:, None]
    return answer


def _exact_attention(case, state):
    """Sequence by sequence and head by head, every row against the list of the positions that it sees."""
    q = state["q"]
    S, L, H, d = q.shape
    Hkv = HEADS[case["heads"]][1]
    out = torch.zeros((S, L, H, d), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((S, L, H), dtype=torch.float64, device=DEVICE)
    table = _values(case["format"])
    for u in range(S // case["drafts"]):
        n = case["length"] if state["lens"] is None else int(state["lens"][u])
        position = torch.arange(n, device=DEVICE)
        at = _at(case, position)
        for g in range(Hkv):
            k, v = (table[state["codes"][u, g].reshape(-1)[at[i]].long()] * state["scales"][u, g, position // case["block"], i].double()[:, None]
                    for i in (0, 1))
            heads = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
            for s in range(u * case["drafts"], (u + 1) * case["drafts"]):
                keys, values = k, v
                if state["k"] is not None:
                    keys, values = torch.cat([k, state["k"][s, :, g].double()]), torch.cat([v, state["v"][s, :, g].double()])
                x = q[s, :, heads].double().reshape(-1, d).mm(keys.t().contiguous()) / float(d) ** 0.5
                z = x.logsumexp(-1)
                out[s, :, heads] = (x - z[:, None]).exp().mm(values).view(L, -1, d)
                lse[s, :, heads] = z.view(L, -1)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    state = prepare(case, seed)
    return {"rotate": _exact_rotation, "store": _exact_store, "attend": _exact_attention}[case["op"]](case, state)
