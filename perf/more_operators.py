"""Timed cases of a key/value cache held in 4 bits, and of low-rank adapters beside the shared 4-bit projections.

A case is a dict of plain values.  "kind" says which operator it times:
  store   rotary embedding of queries and new keys; keys and values go into the 4-bit pages of their sequences and are read back
  attend  attention of new tokens over 4-bit pages (one token or a chunk per sequence; with a window and first tokens that stay)
  project a projection with shared 4-bit weights, and beside it each row's own low-rank adapter
  gated   the gate and the up projection with their adapters, silu(gate) * up

Layer shapes are those of the other timed cases (7B-, 8B-GQA- and 13B-shaped decoder layers, and a generic one with 64-wide heads).
`run` computes a case in elementary torch operations, in 32 bits (64 where a key's rounding to 4 bits hangs on it); with `own` set it
calls the framework's operators.  Places of a page that hold no token have a NaN scale.

A page of the 4-bit cache holds for each key/value head the codes of its tokens and then a 32-bit word per token, scale | zero << 16, with the
scale in the cache's 16-bit type; code c stands for (c - zero) * scale.  Codes of keys: word w of a token has columns 8 w + 2 i at bits 4 i and
8 w + 2 i + 1 at bits 16 + 4 i.  Codes of values: tokens by fours, word 2 Q + p of a four has columns 4 Q + i of its token 2 p at bits 4 i and of
its token 2 p + 1 at bits 16 + 4 i.
"""
import math

import torch

own = False

# heads, key/value heads, head size, hidden size, inner size of the gated block
SHAPES = {"7b": (32, 32, 128, 4096, 11008), "8b_gqa": (32, 8, 128, 4096, 14336), "13b": (40, 40, 128, 5120, 13824), "d64_gqa": (32, 8, 64, 2048, 5504)}
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
MOST_BYTES = 1.2e9                                               # of a drawn case: what the largest listed ones move ...
MOST_FLOPS = 5.0e11                                              # ... and compute


def _store(shape, dtype, page, seqs, tokens, cached, layout="half", share=1.0, late=0):
    return dict(kind="store", shape=shape, dtype=dtype, page=page, seqs=seqs, tokens=tokens, cached=cached, layout=layout, share=share, late=late)


def _attend(shape, dtype, page, seqs, tokens, cached, ragged=False, window=0, sinks=0):
    return dict(kind="attend", shape=shape, dtype=dtype, page=page, seqs=seqs, tokens=tokens, cached=cached, ragged=ragged,
                window=window, sinks=sinks)


def _linear(kind, n_in, n_out, group, rows, run, adapters, rank, bare=0.0):
    """run: rows next to each other that belong to one request; bare: share of the requests that have no adapter."""
    return dict(kind=kind, n_in=n_in, n_out=n_out, group=group, rows=rows, run=run, adapters=adapters, rank=rank, bare=bare)


def listed():
    return [
        # a serving batch's decode step: the new token of each sequence
        dict(name="store_decode_64_7b", **_store("7b", "fp16", 64, 64, 1, 1000)),
        # the next pieces of long prompts: interleaved pairs, half of the head
        dict(name="store_chunk_3x1700_gqa", **_store("8b_gqa", "bf16", 128, 3, 1700, 900, "interleaved", 0.5, 60000)),
        # one user in a chat, a short context in small pages: the smallest call
        dict(name="attend_1x700_gqa", **_attend("8b_gqa", "fp16", 16, 1, 1, 700)),
        # an ordinary decode batch of sequences of all ages
        dict(name="attend_33x3000_gqa", **_attend("8b_gqa", "bf16", 64, 33, 1, 3000, ragged=True)),
        # a large decode batch, one query head per key/value head: the longest stream
        dict(name="attend_64x4000_7b", **_attend("7b", "fp16", 64, 64, 1, 4000)),
        # long chats under a window, a few drafted tokens each, 64-wide heads: four first tokens and the last 1024 are seen
        dict(name="attend_48x4_on_9000_window", **_attend("d64_gqa", "fp16", 32, 48, 4, 9000, ragged=True, window=1024, sinks=4)),
        # a question of 500 tokens about a long document
        dict(name="attend_1x500_on_24000_gqa", **_attend("8b_gqa", "bf16", 128, 1, 500, 24000)),
        # long prompts from the start, the largest products
        dict(name="attend_4x4096_gqa", **_attend("8b_gqa", "fp16", 64, 4, 4096, 0)),
        # three chats with an adapter each: the output projection of a decode step
        dict(name="project_3_7b", **_linear("project", 4096, 4096, 128, 3, 1, 3, 16)),
        # prompts of seven requests, five adapters among them, one request has none: the down projection
        dict(name="project_7x500_gqa", **_linear("project", 14336, 4096, 64, 3500, 500, 5, 32, 0.15)),
        # the decode step of 64 requests with 40 adapters
        dict(name="gated_64_7b", **_linear("gated", 4096, 11008, 128, 64, 1, 40, 16, 0.1)),
        # a batch of short prompts, odd sizes
        dict(name="gated_9x77_13b", **_linear("gated", 5120, 13824, 128, 693, 77, 9, 61)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    pick = rng.random()
    shape, dtype, page = rng.choice(sorted(SHAPES)), rng.choice(sorted(TYPES)), rng.choice([16, 32, 64, 128])
    nh, nkv, d, hidden, inner = SHAPES[shape]
    if pick < 0.2:
        seqs = _log(rng, 1, 64)
        return _store(shape, dtype, page, seqs, _log(rng, 1, 6000 // seqs), _log(rng, 1, 3000), rng.choice(["half", "interleaved"]),
                      rng.choice([1.0, 0.75, 0.5, 0.25]), rng.choice([0, 60000]))
    window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 100, 3000), 0), (_log(rng, 100, 3000), rng.randint(1, 80))])
    token_bytes = 2 * nkv * (d // 2 + 4)
    if pick < 0.45:
        seqs = _log(rng, 1, 160)
        room = MOST_BYTES / token_bytes / seqs
        return _attend(shape, dtype, page, seqs, rng.choice([1, 1, 1, rng.randint(2, 9)]), _log(rng, 40, min(30000, room)),
                       rng.random() < 0.6, window, sinks)
    if pick < 0.65:
        seqs = _log(rng, 1, 12)
        tokens = _log(rng, 10, 4096 // seqs if seqs > 4 else 4096)
        room = min(0.8 * MOST_FLOPS / (4.0 * nh * d * tokens * seqs), MOST_BYTES / (token_bytes * seqs)) - tokens   # (long ones may meet long ones)
        cached = _log(rng, 1, min(24000 if tokens <= 512 else 4096, room)) if room > 1 and rng.random() < 0.7 else 0
        return _attend(shape, dtype, page, seqs, tokens, cached, rng.random() < 0.6, window, sinks)
    kind = rng.choice(["project", "gated"])
    n_in, n_out = (hidden, inner) if kind == "gated" else rng.choice([(hidden, hidden), (inner, hidden), (hidden, (nh + 2 * nkv) * d)])
    if rng.random() < 0.3:                                       # odd sizes, in steps of 8
        n_in, n_out = 8 * _log(rng, 4, n_in // 8), 8 * _log(rng, 1, n_out // 8)
    most = min(4000, 0.9 * MOST_FLOPS / (2.0 * n_in * n_out * (2 if kind == "gated" else 1)))
    per = rng.choice([1, 1, rng.randint(2, 5), _log(rng, 10, 900)])
    seqs = _log(rng, 1, max(1, min(150, most // per)))
    return _linear(kind, n_in, n_out, rng.choice([32, 64, 128]), seqs * per, per, rng.randint(1, min(64, seqs)), _log(rng, 1, 128),
                   rng.choice([0.0, 0.0, 0.2]))


# ---- sizes that follow from a case -------------------------------------------------------------------------------
def _spread(n, count, ragged):
    """`count` lengths: all n, or spread evenly from n / 2 to 3 n / 2 (the same total whatever the order)."""
    if not ragged or count == 1 or n <= 1:
        return [n] * count
    return [max(1, n // 2 + (n * i) // (count - 1)) for i in range(count)]


def _lengths(case, seed=None):
    """New tokens and cached tokens of each sequence (store, attend)."""
    ragged = case.get("ragged", True)
    new, old = _spread(case["tokens"], case["seqs"], ragged), _spread(case["cached"], case["seqs"], ragged)
    if seed is not None:                                          # which sequence is the long one changes with the inputs
        g = torch.Generator().manual_seed(int(seed) % (1 << 62))
        new = [new[i] for i in torch.randperm(len(new), generator=g).tolist()]
        old = [old[i] for i in torch.randperm(len(old), generator=g).tolist()]
    return new, old


def _seen(case, new, old):
    """(query, key) pairs that are visible, and the distinct keys that a call has to read."""
    window, sinks = case["window"], case["sinks"]
    pairs = keys = 0
    for n, o in zip(new, old):
        if not window:
            pairs += n * o + n * (n + 1) // 2
            keys += o + n
            continue
        p = torch.arange(o, o + n, dtype=torch.float64)
        first = (p + 1 - window).clamp(min=0)                     # the window's first key
        pairs += int((p + 1 - first + torch.minimum(first, torch.tensor(float(sinks)).double())).sum())
        lo = max(0, o + 1 - window)
        keys += o + n - lo + min(lo, sinks)
    return pairs, keys


def _matrices(case):
    return 2 if case["kind"] == "gated" else 1


def work(case):
    if case["kind"] in ("project", "gated"):
        K, N, M, r, m = case["n_in"], case["n_out"], case["rows"], case["rank"], _matrices(case)
        weights = N * K // 2 + 4 * N * -(-K // case["group"])
        adapters = min(case["adapters"], M) * 2 * r * (K + N)
        return {"bytes": m * (weights + adapters) + 2 * M * (K + N), "flops": m * 2 * M * (N * K + r * (K + N))}
    nh, nkv, d = SHAPES[case["shape"]][:3]
    new, old = _lengths(case)
    if case["kind"] == "store":
        T = sum(new)
        return {"bytes": T * (4 * nh * d + 4 * nkv * d + 2 * nkv * (d // 2 + 4) + 4 * nkv * d + 4), "flops": T * (nh + 3 * nkv) * 6 * d}
    pairs, keys = _seen(case, new, old)
    return {"bytes": 2 * keys * nkv * (d // 2 + 4) + 4 * sum(new) * nh * d, "flops": 4 * pairs * nh * d}


# ---- inputs ----------------------------------------------------------------------------------------------------
def _gen(seed, slot, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed((int(seed) * 1000003 + slot * 7919) % (1 << 62))
    return g


def _randn(seed, slot, size, dtype, std=1.0):
    return (torch.randn(*size, generator=_gen(seed, slot), device="cuda", dtype=torch.float32) * std).to(dtype)


def _words(free):
    """Bit i % 32 of word i / 32 = page i is free."""
    n = free.numel()
    bits = torch.nn.functional.pad(free.to(torch.int64), (0, -n % 32)).view(-1, 32)
    words = (bits << torch.arange(32, device=free.device)).sum(1)
    return (words - ((words >> 31) << 32)).to(torch.int32)


def _table(case, seed):
    """Slots of the sequences, page table, lengths."""
    new, old = _lengths(case, seed)
    page, B = case["page"], case["seqs"]
    g = torch.Generator().manual_seed((int(seed) * 17 + 3) % (1 << 62))
    n_slots = B + 2
    slots = torch.randperm(n_slots, generator=g)[:B]
    total = [o + n for o, n in zip(old, new)]
    held = [-(-t // page) for t in total]
    n_pages = sum(total) // page + B + 3                          # (the same for every seed)
    order = torch.randperm(n_pages, generator=g).int()
    table = torch.full((1, n_slots, -(-(max(new) + max(old)) // page) + 1), -1, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[0, slots[b], : held[b]] = order[at: at + held[b]]
        at += held[b]
        if case.get("window"):                                   # pages that no query of the call can see are gone
            for j in range(held[b]):
                if (j + 1) * page <= old[b] + 1 - case["window"] and j * page >= case["sinks"]:
                    table[0, slots[b], j] = -1
    length = torch.zeros(1, n_slots, dtype=torch.int32)
    cap = torch.zeros(1, n_slots, dtype=torch.int32)
    length[0, slots] = torch.tensor(total, dtype=torch.int32)
    cap[0, slots] = torch.tensor(held, dtype=torch.int32) * page
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[table[table >= 0].long()] = 1
    refs = refs.cuda()
    offs = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int()
    rows = torch.full((B, max(new)), sum(new), dtype=torch.int64)  # row of a sequence's i-th new token (past the last: one that is not there)
    for b in range(B):
        rows[b, : new[b]] = torch.arange(int(offs[b]), int(offs[b]) + new[b])
    return dict(new=new, old=old, max_new=max(new), max_len=max(total), n_pages=n_pages, table=table.cuda(), kv_len=length.cuda(), kv_cap=cap.cuda(),
                refs=refs, bits=_words(refs == 0), slots=slots.int().cuda(), offs=offs.cuda(), first=torch.tensor(old, dtype=torch.int32).cuda(), rows=rows.cuda())


def _held_tokens(s, page):
    """[n_pages, page]: whether a page's place holds a token of a sequence."""
    P = s["table"].shape[2]
    token = torch.arange(P * page, device="cuda").view(1, P, page)
    inside = token < s["kv_len"][0].view(-1, 1, 1)
    held = torch.zeros(s["n_pages"] + 1, page, dtype=torch.bool, device="cuda")
    held[s["table"][0].long().flatten()] = inside.reshape(-1, page)   # (entries of -1 land in the row past the end)
    return held[: s["n_pages"]]


def _pool(seed, slot, s, case):
    """Pages of codes and scales as a cache of ordinary activations has them: [n_pages, nkv, page * (d / 2 + 4)] bytes."""
    nh, nkv, d = SHAPES[case["shape"]][:3]
    page, dtype = case["page"], TYPES[case["dtype"]]
    g = _gen(seed, slot)
    pool = torch.randint(0, 256, (s["n_pages"], nkv, page * (d // 2 + 4)), generator=g, device="cuda", dtype=torch.uint8)
    scale = (0.4 * torch.exp(0.3 * torch.randn(s["n_pages"], nkv, page, generator=g, device="cuda"))).to(dtype)
    scale.masked_fill_(~_held_tokens(s, page)[:, None], float("nan"))
    zero = torch.randint(4, 12, scale.shape, generator=g, device="cuda", dtype=torch.int16)
    pool[:, :, page * d // 2:] = torch.stack([scale.view(torch.int16), zero], 3).reshape(s["n_pages"], nkv, -1).view(torch.uint8)
    return pool


def _rotary(case):
    return 2 * int(case["share"] * SHAPES[case["shape"]][2] / 2)


def _cache_state(case, seed):
    nh, nkv, d = SHAPES[case["shape"]][:3]
    dtype = TYPES[case["dtype"]]
    s = _table(case, seed)
    s["case"], T = case, sum(s["new"])
    s["k"], s["v"] = _pool(seed, 1, s, case), _pool(seed, 4, s, case)
    s["out"] = torch.empty(T, nh, d, dtype=dtype, device="cuda")
    if case["kind"] == "attend":
        s["q"] = _randn(seed, 2, (T, nh, d), dtype)
        return s
    # what the q|k|v product leaves, one row per token; a few columns of the keys are far larger than the others, as they are in earnest
    qkv = torch.randn(T, nh + 2 * nkv, d, generator=_gen(seed, 2), device="cuda")
    qkv[:, nh: nh + nkv] *= torch.exp(0.7 * torch.randn(nkv, d, generator=_gen(seed, 5), device="cuda"))
    s["qkv"] = qkv.to(dtype)
    # a sequence's tokens at this layer are some of its positions: steps of 1 to 3
    steps = torch.randint(1, 4, (T,), generator=_gen(seed, 3), device="cuda")
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), torch.tensor(s["new"], device="cuda"))
    run_up = steps.cumsum(0)
    begin = torch.cat([run_up.new_zeros(1), run_up])[s["offs"].long()][seq]
    s["positions"] = (s["first"].long()[seq] + run_up - begin + case["late"]).int()
    rd = _rotary(case)
    s["freqs"] = (10000.0 ** (-2.0 * torch.arange(rd // 2, dtype=torch.float64) / rd)).cuda()
    s["k_new"], s["v_new"] = (torch.empty(T, nkv, d, dtype=dtype, device="cuda") for _ in range(2))
    return s


def _linear_state(case, seed):
    K, N, M, r, n = case["n_in"], case["n_out"], case["rows"], case["rank"], case["adapters"]
    g = _gen(seed, 1)
    s = dict(case=case, x=_randn(seed, 2, (M, K), torch.float16), parts=[])
    seqs = -(-M // case["run"])
    # every adapter is in use, by the requests in no order
    ids = torch.cat([torch.arange(n), torch.randint(0, n, (seqs - n,), generator=torch.Generator().manual_seed(int(seed) % (1 << 62)))])
    bare = torch.rand(seqs, generator=torch.Generator().manual_seed((int(seed) + 1) % (1 << 62))) < case["bare"]
    ids = torch.where(bare, -1, ids)[torch.randperm(seqs, generator=torch.Generator().manual_seed((int(seed) + 2) % (1 << 62)))]
    s["ids"] = ids.repeat_interleave(case["run"])[:M].int().cuda()
    for i in range(_matrices(case)):
        p = dict(codes=torch.randint(-(1 << 31), 1 << 31, (N, K // 8), generator=g, device="cuda", dtype=torch.int64).int())
        groups = -(-K // case["group"])
        p["scales"] = (0.7 / math.sqrt(K) / 4.6 * 1.5 * (0.5 + torch.rand(N, groups, generator=g, device="cuda"))).half()
        p["zeros"] = torch.randint(5, 11, (N, groups), generator=g, device="cuda").half()
        p["down"] = _randn(seed, 10 + i, (n, r, K), torch.float16, 1.0 / math.sqrt(K))
        p["up"] = _randn(seed, 20 + i, (n, N, r), torch.float16, 0.3 / math.sqrt(r))
        # adapters of one pool have ranks of their own, up to the pool's
        p["rank"] = torch.randint((r + 1) // 2, r + 1, (n,), generator=g, device="cuda").int()
        p["rank"][0] = r
        p["scale"] = 0.5 + torch.rand(n, generator=g, device="cuda")
        s["parts"].append(p)
    s["out"] = torch.empty(M, N, dtype=torch.float16, device="cuda")
    return s


def _state(case, seed):
    return (_linear_state if case["kind"] in ("project", "gated") else _cache_state)(case, seed)


def prepare(case, seed):
    s = _state(case, seed)
    if own:                                                       # the framework's handles on these arrays, and what a program keeps beside them
        import paper_2602_10431_amd as qt
        if case["kind"] in ("project", "gated"):
            for p in s["parts"]:
                p["linear"] = qt.qtale_prepack(p["codes"], p["scales"], p["zeros"], case["n_out"], case["n_in"], 4, case["group"])
                p["lora"] = qt.Lora(p["down"], p["up"], p["rank"], p["scale"])
            s["workspace"] = qt.alloc_lora_workspace([p["lora"] for p in s["parts"]], case["rows"])
        else:
            d = SHAPES[case["shape"]][2]
            kv = s["kv"] = qt.PagedKV(s["k"], s["v"], s["refs"], s["bits"], s["table"], s["kv_len"], s["kv_cap"], dtype=TYPES[case["dtype"]], head_dim=d)
            if case["kind"] == "store":
                s["rope"] = qt.Rope(_rotary(case), 10000.0, case["layout"])
            else:
                s["workspace"] = qt.alloc_paged_workspace(kv, SHAPES[case["shape"]][0], sum(s["new"]), case["seqs"], s["max_new"], s["max_len"])
    return s


# ---- one pass --------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return {"store": _own_store, "attend": _own_attend, "project": _own_project, "gated": _own_gated}[state["case"]["kind"]](state)
    return {"store": _plain_store, "attend": _plain_attend, "project": _plain_project, "gated": _plain_gated}[state["case"]["kind"]](state)


def _own_store(s):
    import paper_2602_10431_amd as qt
    nh, nkv, d = SHAPES[s["case"]["shape"]][:3]
    q, k, v = s["qkv"].split((nh, nkv, nkv), 1)
    qt.qtale_paged_rope_append(s["kv"], 0, s["rope"], q, k, v, s["offs"], s["positions"], first=s["first"], slots=s["slots"], q_out=s["out"])
    qt.qtale_paged_read(s["kv"], 0, s["offs"], s["first"], slots=s["slots"], k_out=s["k_new"], v_out=s["v_new"])
    return dict(q=s["out"], k=s["k_new"], v=s["v_new"])


def _own_attend(s):
    import paper_2602_10431_amd as qt
    c = s["case"]
    return qt.qtale_paged_attention(s["kv"], 0, s["q"], s["offs"], first=s["first"], slots=s["slots"], out=s["out"], window=c["window"],
                                    sinks=c["sinks"], max_new=s["max_new"], max_len=s["max_len"], workspace=s["workspace"])


def _own_project(s):
    import paper_2602_10431_amd as qt
    p = s["parts"][0]
    return qt.qtale_linear_lora_w4a16(p["linear"], p["lora"], s["x"], s["ids"], out=s["out"], workspace=s["workspace"])


def _own_gated(s):
    import paper_2602_10431_amd as qt
    g, u = s["parts"]
    return qt.qtale_swiglu_lora_w4a16(g["linear"], u["linear"], g["lora"], u["lora"], s["x"], s["ids"], out=s["out"], workspace=s["workspace"])


def _turn(t, cos, sin, layout, rd):
    """Rotates the first rd columns of t [T, heads, d]; cos, sin [T, 1, rd / 2]."""
    out = t.clone()
    if layout == "half":
        a, b = t[..., : rd // 2], t[..., rd // 2: rd]
        out[..., : rd // 2], out[..., rd // 2: rd] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = t[..., 0:rd:2], t[..., 1:rd:2]
        out[..., 0:rd:2], out[..., 1:rd:2] = a * cos - b * sin, b * cos + a * sin
    return out


def _in_4_bits(x):
    """The values that rows of x (16-bit) are held as."""
    w = x.double()
    lo, hi = w.amin(-1, keepdim=True).clamp(max=0.0), w.amax(-1, keepdim=True).clamp(min=0.0)
    scale = ((hi - lo) / 15.0).to(x.dtype).double()
    scale = torch.where(scale == 0.0, 1.0, scale)
    zero = torch.round(-lo / scale).clamp(max=15.0)
    code = (torch.round(w / scale) + zero).clamp(0.0, 15.0)
    return ((code - zero) * scale).to(x.dtype)


def _plain_store(s):
    c = s["case"]
    nh, nkv, d = SHAPES[c["shape"]][:3]
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    q, k, v = s["qkv"].split((nh, nkv, nkv), 1)
    s["out"].copy_(_turn(q.double(), cos, sin, c["layout"], _rotary(c)))
    s["k_new"].copy_(_in_4_bits(_turn(k.double(), cos, sin, c["layout"], _rotary(c)).to(k.dtype)))
    s["v_new"].copy_(_in_4_bits(v))
    return dict(q=s["out"], k=s["k_new"], v=s["v_new"])


def _plain_attend(s):
    c = s["case"]
    nh, nkv, d = SHAPES[c["shape"]][:3]
    page, B = c["page"], c["seqs"]
    P = -(-s["max_len"] // page)
    n, n_new, rep = P * page, s["max_new"], nh // nkv
    ids = s["table"][0][s["slots"].long(), :P].long()             # [B, P]
    shifts = torch.arange(0, 16, 4, device="cuda", dtype=torch.int32)

    def values(pool, keys):
        rows = pool[ids.clamp(min=0)]                             # [B, P, nkv, bytes]
        codes, params = rows[..., : page * d // 2].contiguous().view(torch.int16), rows[..., page * d // 2:].contiguous().view(torch.int16)
        codes = (codes[..., None].int() >> shifts) & 15           # [B, P, nkv, 16-bit pieces, 4]
        if keys:                                                  # pieces: token, word, parity of the column
            codes = codes.view(B, P, nkv, page, d // 8, 2, 4).transpose(5, 6)
        else:                                                     # pieces: four, column / 4, pair, token of the pair
            codes = codes.view(B, P, nkv, page // 4, d // 4, 2, 2, 4).permute(0, 1, 2, 3, 5, 6, 4, 7)
        codes = codes.reshape(B, P, nkv, page, d).float()
        params = params.view(B, P, nkv, page, 2)
        scale, zero = params[..., 0].contiguous().view(TYPES[c["dtype"]]).float(), params[..., 1].float()
        return ((codes - zero[..., None]) * scale[..., None]).transpose(1, 2).reshape(B, nkv, n, d)

    key = torch.arange(n, device="cuda")
    there = (ids >= 0).repeat_interleave(page, 1) & (key < s["kv_len"][0][s["slots"].long()].long()[:, None])   # [B, n]
    k, v = (values(s[x], x == "k").masked_fill(~there[:, None, :, None], 0.0) for x in ("k", "v"))
    q = torch.cat([s["q"], s["q"].new_zeros(1, nh, d)])[s["rows"]].float()   # [B, n_new, nh, d]
    q = q.view(B, n_new, nkv, rep, d).permute(0, 2, 3, 1, 4).reshape(B * nkv, rep * n_new, d)
    place = (s["first"].long()[:, None] + torch.arange(n_new, device="cuda"))[:, :, None]
    seen = there[:, None] & (key <= place)
    if c["window"]:
        seen &= (key > place - c["window"]) | (key < c["sinks"])
    score = torch.bmm(q, k.view(B * nkv, n, d).transpose(1, 2).contiguous()).view(B, nkv * rep, n_new, n).mul_(d ** -0.5)
    score = score.masked_fill_(~seen[:, None], float("-inf"))
    p = torch.exp_(score.sub_(score.amax(3, keepdim=True).clamp(min=-1e30)))
    p = p.div_(p.sum(3, keepdim=True).clamp(min=1e-30)).view(B * nkv, rep * n_new, n)
    o = torch.bmm(p, v.view(B * nkv, n, d)).view(B, nkv, rep, n_new, d).permute(0, 3, 1, 2, 4).reshape(B * n_new, nh, d)
    held = s["rows"].flatten() < s["out"].shape[0]
    s["out"].copy_(o[held])                                       # (rows in order of sequences)
    return s["out"]


def _plain_linear(s, p):
    c = s["case"]
    n, r, K = p["down"].shape
    x = s["x"].float()
    codes = ((p["codes"][..., None] >> torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)) & 15).view(c["n_out"], K).float()
    spread = lambda t: t.float().repeat_interleave(c["group"], 1)[:, :K]
    y = x @ ((codes - spread(p["zeros"])) * spread(p["scales"])).t()
    # all adapters' inner values of all rows; a row keeps those of its own
    inner = (x @ p["down"].float().view(n * r, K).t()).view(-1, n, r)
    keep = (s["ids"][:, None] == torch.arange(n, device="cuda"))[:, :, None] & (torch.arange(r, device="cuda") < p["rank"][:, None])
    inner = torch.where(keep, inner * p["scale"][:, None], 0.0).view(-1, n * r)
    return y + inner @ p["up"].float().transpose(1, 2).reshape(n * r, -1)


def _plain_project(s):
    s["out"].copy_(_plain_linear(s, s["parts"][0]))
    return s["out"]


def _plain_gated(s):
    g, u = (_plain_linear(s, p) for p in s["parts"])
    s["out"].copy_(g / (1.0 + torch.exp(-g)) * u)
    return s["out"]


# ---- the same results in 64 bits ------------------------------------------------------------------------------
def _exact_rows(x):
    """Rows quantized to 4 bits, as the values they stand for, in 64 bits."""
    t, x = x.dtype, x.double()
    low = torch.minimum(x.min(dim=-1).values, torch.zeros((), dtype=torch.float64, device=x.device))
    high = torch.maximum(x.max(dim=-1).values, torch.zeros((), dtype=torch.float64, device=x.device))
    step = torch.div(high - low, 15).to(t).double()
    step[step == 0] = 1.0
    origin = torch.round(low / step).neg().clamp(max=15)
    level = torch.round(x / step[..., None]).add(origin[..., None]).clamp(min=0, max=15)
    return (level - origin[..., None]) * step[..., None]


def _exact_entries(pool, case, page_ids, keys):
    """[entries of the pages, nkv, d] in 64 bits, code by code from its bits."""
    d, page = SHAPES[case["shape"]][2], case["page"]
    rows = pool[page_ids]
    n, nkv = rows.shape[:2]
    byte = rows[..., : page * d // 2].long()
    word = (byte.view(n, nkv, -1, 4) << torch.tensor([0, 8, 16, 24], device="cuda")).sum(3)
    t, col = torch.arange(page, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    if keys:
        at, shift = t * (d // 8) + col // 8, 16 * (col % 2) + 4 * ((col % 8) // 2)
    else:
        at, shift = (t // 4) * (d // 2) + 2 * (col // 4) + (t % 4) // 2, 16 * (t % 2) + 4 * (col % 4)
    code = (word[:, :, at] >> shift) & 15                         # [n, nkv, page, d]
    param = rows[..., page * d // 2:].contiguous().view(torch.int16).view(n, nkv, page, 2)
    step = param[..., :1].contiguous().view(TYPES[case["dtype"]]).double()
    return ((code - param[..., 1:].long()).double() * step).transpose(1, 2).reshape(n * page, nkv, d)


def exact(case, seed):
    s = _state(case, seed)
    if case["kind"] in ("project", "gated"):
        ys = []
        for p in s["parts"]:
            K, x = case["n_in"], s["x"].double()
            nibble = torch.stack([(p["codes"] >> (4 * j)) & 15 for j in range(8)], 2).flatten(1)
            column = torch.arange(K, device="cuda") // case["group"]
            y = x @ ((nibble - p["zeros"].long()[:, column]).double() * p["scales"].double()[:, column]).t()
            for a in range(case["adapters"]):
                rows, r = torch.nonzero(s["ids"] == a)[:, 0], int(p["rank"][a])
                y[rows] += float(p["scale"][a]) * (x[rows] @ p["down"][a, :r].double().t()) @ p["up"][a, :, :r].double().t()
            ys.append(y)
        return ys[0] if len(ys) == 1 else ys[0] * torch.sigmoid(ys[0]) * ys[1]
    nh, nkv, d = SHAPES[case["shape"]][:3]
    page = case["page"]
    if case["kind"] == "store":
        rd = _rotary(case)
        turn = torch.polar(torch.ones(len(s["positions"]), rd // 2, dtype=torch.float64, device="cuda"), torch.outer(s["positions"].double(), s["freqs"]))
        x = s["qkv"].double()
        head = x[:, : nh + nkv, :rd]
        pairs = head.reshape(-1, nh + nkv, rd // 2, 2) if case["layout"] == "interleaved" else head.reshape(-1, nh + nkv, 2, rd // 2).transpose(2, 3)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        x[:, : nh + nkv, :rd] = (z if case["layout"] == "interleaved" else z.transpose(2, 3)).reshape(-1, nh + nkv, rd)
        return dict(q=x[:, :nh].contiguous(), k=_exact_rows(x[:, nh: nh + nkv].to(TYPES[case["dtype"]])), v=_exact_rows(s["qkv"][:, nh + nkv:]))
    out = torch.empty(sum(s["new"]), nh, d, dtype=torch.float64, device="cuda")
    t = 0
    for b, (n, o) in enumerate(zip(s["new"], s["old"])):
        row = s["table"][0, int(s["slots"][b])].tolist()
        at = [(j * page, row[j]) for j in range(-(-(o + n) // page)) if row[j] >= 0]
        where = torch.cat([torch.arange(a, a + page) for a, _ in at]).cuda()
        ids = torch.tensor([p for _, p in at], device="cuda")
        back = torch.arange(o, o + n, device="cuda")[:, None] - where[None]
        hidden = (back < 0) | (where >= o + n)[None]
        if case["window"]:
            hidden |= (back >= case["window"]) & (where >= case["sinks"])[None]
        k, v = _exact_entries(s["k"], case, ids, True), _exact_entries(s["v"], case, ids, False)
        k[where >= o + n] = v[where >= o + n] = 0.0
        for h in range(nh):
            z = (s["q"][t: t + n, h].double() @ k[:, h * nkv // nh].t()) / math.sqrt(d)
            out[t: t + n, h] = torch.softmax(z.masked_fill(hidden, -math.inf), 1) @ v[:, h * nkv // nh]
        t += n
    return out
