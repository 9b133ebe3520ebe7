"""Timed cases of the paged key/value cache: rotary embedding with the append, attention over pages, and the pages themselves.

A case is a dict of plain values.  "kind" says which operator it times:
  rope    rotary embedding of queries and new keys, keys and values written into the pages of their sequences
  attend  attention of new tokens over the pages (one token or a chunk per sequence; with a window and first tokens that stay)
  branch  sequences are forked, then every copy makes room for its next tokens (a shared last page is copied first)
  compact the pages in use move to the front of the pool
  retire  some sequences end, the others drop the pages that their window has left behind

Layer shapes are those of the other timed cases (7B-, 8B-GQA- and 13B-shaped decoder layers, and a generic one with 64-wide heads).
`run` computes a case in elementary torch operations, in 32 bits (positions times frequencies in 64, or the angle of a late position is
lost); with `own` set it calls the framework's operators.  Memory that no sequence holds is NaN where a result could pick it up.
"""
import math

import torch

own = False

# heads, key/value heads, head size
SHAPES = {"7b": (32, 32, 128), "8b_gqa": (32, 8, 128), "13b": (40, 40, 128), "d64_gqa": (32, 8, 64)}
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
MOST_BYTES = 2.2e9                                               # of a drawn case: what the largest listed ones move ...
MOST_FLOPS = 5.5e11                                              # ... and compute


def _rope(shape, dtype, page, seqs, tokens, cached, layout="half", share=1.0, scaling="none", late=0):
    return dict(kind="rope", shape=shape, dtype=dtype, page=page, seqs=seqs, tokens=tokens, cached=cached, layout=layout, share=share,
                scaling=scaling, late=late)


def _attend(shape, dtype, page, seqs, tokens, cached, ragged=False, window=0, sinks=0):
    return dict(kind="attend", shape=shape, dtype=dtype, page=page, seqs=seqs, tokens=tokens, cached=cached, ragged=ragged,
                window=window, sinks=sinks)


def _pages(kind, shape, dtype, page, layers, seqs, cached, copies=1, tokens=1, window=0, sinks=0):
    return dict(kind=kind, shape=shape, dtype=dtype, page=page, layers=layers, seqs=seqs, cached=cached, copies=copies, tokens=tokens,
                window=window, sinks=sinks)


def listed():
    return [
        # a serving batch's decode step: the new token of each sequence
        dict(name="rope_decode_64_7b", **_rope("7b", "fp16", 64, 64, 1, 1000)),
        # the next pieces of long prompts: interleaved pairs, half of the head, a context stretched past its training length
        dict(name="rope_chunk_3x1700_gqa", **_rope("8b_gqa", "bf16", 128, 3, 1700, 900, layout="interleaved", share=0.5,
                                                   scaling="parts", late=60000)),
        # one user in a chat, a short context in small pages: the smallest call
        dict(name="attend_1x700_7b", **_attend("7b", "fp16", 16, 1, 1, 700)),
        # an ordinary decode batch of sequences of all ages
        dict(name="attend_33x3000_gqa", **_attend("8b_gqa", "bf16", 64, 33, 1, 3000, ragged=True)),
        # the decode batch of bench.py, one query head per key/value head
        dict(name="attend_64x2048_7b", **_attend("7b", "fp16", 64, 64, 1, 2048)),
        # long chats under a window: four first tokens and the last 1024 are seen, the pages between are gone
        dict(name="attend_48x9000_window", **_attend("8b_gqa", "fp16", 32, 48, 1, 9000, ragged=True, window=1024, sinks=4)),
        # the next piece of two prompts on top of what is cached, 64-wide heads
        dict(name="attend_2x700_on_1400_d64", **_attend("d64_gqa", "fp16", 32, 2, 700, 1400, ragged=True)),
        # a question of 500 tokens about a long document
        dict(name="attend_1x500_on_24000_gqa", **_attend("8b_gqa", "bf16", 128, 1, 500, 24000)),
        # long prompts from the start, the largest products
        dict(name="attend_4x4096_gqa", **_attend("8b_gqa", "fp16", 64, 4, 4096, 0)),
        # eight prompts, four answers each, all layers: the first step of the answers
        dict(name="branch_32x8x4", **_pages("branch", "8b_gqa", "fp16", 64, 32, 8, 900, copies=4)),
        # after a busy hour: half of the pool's pages are free, scattered
        dict(name="compact_32x8", **_pages("compact", "8b_gqa", "bf16", 64, 32, 8, 1500)),
        # a step's end: a quarter of the sequences have their answer, the rest let go of what their window left
        dict(name="retire_32x64", **_pages("retire", "d64_gqa", "fp16", 32, 32, 64, 2500, window=1024, sinks=4)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    pick = rng.random()
    shape, dtype, page = rng.choice(sorted(SHAPES)), rng.choice(sorted(TYPES)), rng.choice([16, 32, 64, 128])
    nh, nkv, d = SHAPES[shape]
    if pick < 0.2:
        seqs = _log(rng, 1, 64)
        return _rope(shape, dtype, page, seqs, _log(rng, 1, 6000 // seqs), _log(rng, 1, 3000), rng.choice(["half", "interleaved"]),
                     rng.choice([1.0, 0.75, 0.5, 0.25]), rng.choice(["none", "linear", "base", "bands", "parts"]), rng.choice([0, 60000]))
    window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 100, 3000), 0), (_log(rng, 100, 3000), rng.randint(1, 80))])
    if pick < 0.55:
        seqs = _log(rng, 1, 160)
        room = MOST_BYTES / (4.0 * nkv * d) / seqs
        return _attend(shape, dtype, page, seqs, rng.choice([1, 1, 1, rng.randint(2, 9)]), _log(rng, 40, min(30000, room)),
                       rng.random() < 0.6, window, sinks)
    if pick < 0.8:
        seqs = _log(rng, 1, 12)
        tokens = _log(rng, 10, 4096 // seqs if seqs > 4 else 4096)
        room = min(0.8 * MOST_FLOPS / (4.0 * nh * d * tokens * seqs), MOST_BYTES / (4.0 * nkv * d * seqs)) - tokens   # (long ones may meet long ones)
        cached = _log(rng, 1, min(24000 if tokens <= 512 else 4096, room)) if room > 1 and rng.random() < 0.7 else 0
        return _attend(shape, dtype, page, seqs, tokens, cached, rng.random() < 0.6, window, sinks)
    layers, seqs = rng.choice([1, 2, 8, 24, 32]), _log(rng, 1, 40)
    copies = rng.randint(1, 5) if pick < 0.87 else 1
    room = 1.2e9 / (4.0 * nkv * d) / (layers * seqs)
    cached = max(page, min(_log(rng, 100, 4000), int(room)))
    if pick < 0.87:
        case = _pages("branch", shape, dtype, page, layers, seqs, cached, copies, _log(rng, 1, 60))
    elif pick < 0.94:
        case = _pages("compact", shape, dtype, page, layers, seqs, cached)
    else:
        case = _pages("retire", shape, dtype, page, layers, seqs, cached, window=_log(rng, 100, 3000), sinks=rng.choice([0, 4, 40]))
    while 4 * page * nkv * d * _pool_pages(case) > 2e9:
        case["layers" if case["layers"] > case["seqs"] else "seqs"] //= 2
    return case


# ---- sizes that follow from a case -------------------------------------------------------------------------------
def _spread(n, count, ragged):
    """`count` lengths: all n, or spread evenly from n / 2 to 3 n / 2 (the same total whatever the order)."""
    if not ragged or count == 1 or n <= 1:
        return [n] * count
    return [max(1, n // 2 + (n * i) // (count - 1)) for i in range(count)]


def _lengths(case, seed=None):
    """New tokens and cached tokens of each sequence (rope, attend)."""
    ragged = case.get("ragged", True)
    new, old = _spread(case["tokens"], case["seqs"], ragged), _spread(case["cached"], case["seqs"], ragged)
    if seed is not None:                                          # which sequence is the long one changes with the inputs
        g = torch.Generator().manual_seed(int(seed) % (1 << 62))
        new = [new[i] for i in torch.randperm(len(new), generator=g).tolist()]
        old = [old[i] for i in torch.randperm(len(old), generator=g).tolist()]
    return new, old


def _layer_lengths(case, seed=0):
    """[layers][sequences] cached tokens (branch, compact, retire): a layer holds those that executed it, 50 to 100 % of them."""
    g = torch.Generator().manual_seed((int(seed) * 31 + 5) % (1 << 62))
    L, S, n = case["layers"], case["seqs"], case["cached"]
    return (n * (0.5 + 0.5 * torch.rand(L, S, generator=g))).int().clamp(min=1)


def _grow(case):
    """Pages that a sequence's next tokens may need, and one for its last page."""
    return -(-case["tokens"] // case["page"]) + 1


def _pool_pages(case):
    """Pages of the pool (branch, compact, retire), whatever the layers' lengths: about three quarters of `most` are in use at the start."""
    most = case["layers"] * case["seqs"] * -(-case["cached"] // case["page"])
    if case["kind"] == "branch":
        return most + 7 + case["layers"] * case["seqs"] * case["copies"] * _grow(case)
    return most + 7 + (most // 2 if case["kind"] == "compact" else 0)


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


def work(case):
    nh, nkv, d = SHAPES[case["shape"]]
    page_bytes = 4 * case["page"] * nkv * d                       # keys and values of a page
    if case["kind"] == "rope":
        T = sum(_lengths(case)[0])
        return {"bytes": T * (4 * nh * d + 8 * nkv * d + 4), "flops": T * (nh + nkv) * 3 * int(case["share"] * d)}
    if case["kind"] == "attend":
        new, old = _lengths(case)
        pairs, keys = _seen(case, new, old)
        return {"bytes": 4 * keys * nkv * d + 4 * sum(new) * nh * d, "flops": 4 * pairs * nh * d}
    lens = _layer_lengths(case).double()
    held = torch.ceil(lens / case["page"])
    if case["kind"] == "branch":
        filled = float(torch.remainder(lens, case["page"]).sum())  # copied for each copy of a sequence but the last
        return {"bytes": (case["copies"] - 1) * (2 * filled * 4 * nkv * d + 8 * float(held.sum())), "flops": 0}
    if case["kind"] == "compact":                                 # about a half of the pages in use lies in the pool's back half
        return {"bytes": float(held.sum()) / 2 * (2 * page_bytes + 8), "flops": 0}
    return {"bytes": 12 * float(held.sum()) * 0.6, "flops": 0}    # a table entry, its page's count (read and written)


# ---- inputs ----------------------------------------------------------------------------------------------------
def _gen(seed, slot, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed((int(seed) * 1000003 + slot * 7919) % (1 << 62))
    return g


def _randn(seed, slot, size, dtype, std=1.0):
    return (torch.randn(*size, generator=_gen(seed, slot), device="cuda", dtype=torch.float32) * std).to(dtype)


def _pool(seed, n_pages, case):
    nh, nkv, d = SHAPES[case["shape"]]
    g = _gen(seed, 1)
    return [torch.randn(n_pages, nkv, case["page"], d, generator=g, device="cuda", dtype=TYPES[case["dtype"]]) for _ in range(2)]


def _words(free):
    """Bit i % 32 of word i / 32 = page i is free."""
    n = free.numel()
    bits = torch.nn.functional.pad(free.to(torch.int64), (0, -n % 32)).view(-1, 32)
    words = (bits << torch.arange(32, device=free.device)).sum(1)
    return (words - ((words >> 31) << 32)).to(torch.int32)


def _one_layer(case, seed):
    """Everything of a rope or attend case but the pool's contents: slots of the sequences, page table, lengths."""
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
    offs = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int()
    return dict(new=new, old=old, max_new=max(new), max_len=max(total), n_pages=n_pages, table=table.cuda(), kv_len=length.cuda(), kv_cap=cap.cuda(), refs=refs.cuda(),
                slots=slots.int().cuda(), offs=offs.cuda(), first=torch.tensor(old, dtype=torch.int32).cuda())


def _held_tokens(s, page):
    """[n_pages, page]: whether a page's place holds a token of a sequence."""
    P = s["table"].shape[2]
    token = torch.arange(P * page, device="cuda").view(1, P, page)
    inside = token < s["kv_len"][0].view(-1, 1, 1)
    held = torch.zeros(s["n_pages"] + 1, page, dtype=torch.bool, device="cuda")
    held[s["table"][0].long().flatten()] = inside.reshape(-1, page)   # (entries of -1 land in the row past the end)
    return held[: s["n_pages"]]


SCALING = {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=4.0),
           "bands": dict(factor=8.0, original_len=8192, low=1.0, high=4.0), "parts": dict(factor=16.0, original_len=4096, low=1.0, high=32.0)}


def _rotary(case):
    return 2 * int(case["share"] * SHAPES[case["shape"]][2] / 2)


def _frequencies(case):
    """Angle per position of every pair (float64), and the factor on cos and sin."""
    rd, how = _rotary(case), SCALING[case["scaling"]]
    base = 10000.0
    i = torch.arange(rd // 2, dtype=torch.float64)
    if case["scaling"] == "base":
        base *= how["factor"] ** (rd / (rd - 2))
    f = base ** (-2.0 * i / rd)
    if case["scaling"] == "linear":
        return f / how["factor"], 1.0
    if case["scaling"] == "bands":
        turns = how["original_len"] * f / (2 * math.pi)            # of the pair over the original length
        keep = ((turns - how["low"]) / (how["high"] - how["low"])).clamp(0, 1)
        return f * (keep + (1 - keep) / how["factor"]), 1.0
    if case["scaling"] == "parts":
        where = lambda turns: rd * math.log(how["original_len"] / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(where(how["high"]))), min(rd - 1, math.ceil(where(how["low"])))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / how["factor"] * ramp, 0.1 * math.log(how["factor"]) + 1.0
    return f, 1.0


def _state(case, seed):
    nh, nkv, d = SHAPES[case["shape"]]
    dtype, page = TYPES[case["dtype"]], case["page"]
    if case["kind"] in ("rope", "attend"):
        s = _one_layer(case, seed)
        s["case"], T = case, sum(s["new"])
        s["k"], s["v"] = _pool(seed, s["n_pages"], case)
        s["bits"] = _words(s["refs"] == 0)
        s["out"] = torch.empty(T, nh, d, dtype=dtype, device="cuda")
        if case["kind"] == "rope":
            # what the q|k|v product leaves: one row per token
            s["qkv"] = _randn(seed, 2, (T, nh + 2 * nkv, d), dtype)
            # a sequence's tokens at this layer are some of its positions: steps of 1 to 3
            steps = torch.randint(1, 4, (T,), generator=_gen(seed, 3), device="cuda")
            seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), torch.tensor(s["new"], device="cuda"))
            run_up = steps.cumsum(0)
            begin = torch.cat([run_up.new_zeros(1), run_up])[s["offs"].long()][seq]
            s["positions"] = (s["first"].long()[seq] + run_up - begin + case["late"]).int()
            s["freqs"], s["magnitude"] = _frequencies(case)
            s["freqs"] = s["freqs"].cuda()
        else:
            stale = ~_held_tokens(s, page)[:, None, :, None]
            for t in (s["k"], s["v"]):
                t.masked_fill_(stale, float("nan"))
            s["q"] = _randn(seed, 2, (T, nh, d), dtype, 2.0)
        return s

    # branch, compact, retire: the pages of all layers come from one pool
    lens = _layer_lengths(case, seed)
    L, S, copies = case["layers"], case["seqs"], case["copies"]
    g = torch.Generator().manual_seed((int(seed) * 13 + 1) % (1 << 62))
    n_slots = S * copies + 1
    slots = torch.randperm(n_slots, generator=g)
    held = -(-lens // page)
    live = int(held.sum())
    n_pages = _pool_pages(case)
    max_pages = -(-case["cached"] // page) + _grow(case)
    order = torch.randperm(n_pages, generator=g)[:live].int()
    table = torch.full((L, n_slots, max_pages), -1, dtype=torch.int32)
    place = torch.arange(max_pages).view(1, 1, -1) < held.unsqueeze(2)
    rows = torch.full((L, S, max_pages), -1, dtype=torch.int32)
    rows[place] = order
    table[:, slots[:S]] = rows
    kv_len, kv_cap = torch.zeros(L, n_slots, dtype=torch.int32), torch.zeros(L, n_slots, dtype=torch.int32)
    kv_len[:, slots[:S]] = lens
    kv_cap[:, slots[:S]] = held * page
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[order.long()] = 1
    # the bookkeeping lies in one buffer: a pass first puts it back to where the case begins
    parts = [t.cuda() for t in (table, kv_len, kv_cap, refs, _words(refs == 0))]
    staged = torch.cat([t.flatten() for t in parts])
    now = torch.empty_like(staged)
    s = dict(case=case, staged=staged, now=now)
    at = 0
    for name, t in zip(("table", "kv_len", "kv_cap", "refs", "bits"), parts):
        s[name] = now[at: at + t.numel()].view(t.shape)
        at += t.numel()
    s["k"], s["v"] = _pool(seed, n_pages, case)
    s["n_pages"] = n_pages
    now.copy_(staged)
    if case["kind"] == "branch":
        s["src"] = slots[:S].repeat_interleave(copies - 1).int().cuda()
        s["dst"] = slots[S: S * copies].int().cuda()
        s["slots"] = slots[: S * copies].int().cuda()
        s["offs"] = torch.arange(0, S * copies + 1, dtype=torch.int32).cuda() * case["tokens"]
    elif case["kind"] == "retire":
        ended = max(1, S // 4)
        s["ended"], s["going"] = slots[:ended].int().cuda(), slots[ended:S].int().cuda()
    return s


def prepare(case, seed):
    s = _state(case, seed)
    if own:                                                       # the framework's handle on the pool, and what a program keeps beside it
        import paper_2602_10431_amd as qt
        kv = s["kv"] = qt.PagedKV(s["k"], s["v"], s["refs"], s["bits"], s["table"], s["kv_len"], s["kv_cap"])
        if case["kind"] == "rope":
            s["rope"] = qt.Rope(_rotary(case), 10000.0, case["layout"], case["scaling"], **SCALING[case["scaling"]])
        elif case["kind"] == "attend":
            s["workspace"] = qt.alloc_paged_workspace(kv, SHAPES[case["shape"]][0], sum(s["new"]), case["seqs"], s["max_new"],
                                                      s["max_len"])
        else:
            B = case["seqs"] * case["copies"]
            s["workspace"] = qt.alloc_pages_workspace(kv, B)
            s["first"] = torch.empty(case["layers"], B, dtype=torch.int32, device="cuda")
            s["missing"], s["n_live"] = (torch.empty(1, dtype=torch.int32, device="cuda") for _ in range(2))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if case["kind"] in ("branch", "compact", "retire"):
        state["now"].copy_(state["staged"])
        return (_own_pages if own else _plain_pages)(state)
    if case["kind"] == "rope":
        return (_own_rope if own else _plain_rope)(state)
    return (_own_attend if own else _plain_attend)(state)


def _own_rope(s):
    import paper_2602_10431_amd as qt
    nh, nkv, d = SHAPES[s["case"]["shape"]]
    q, k, v = s["qkv"].split((nh, nkv, nkv), 1)
    qt.qtale_paged_rope_append(s["kv"], 0, s["rope"], q, k, v, s["offs"], s["positions"], first=s["first"], slots=s["slots"], q_out=s["out"])
    return dict(q=s["out"], k=s["k"], v=s["v"])


def _own_attend(s):
    import paper_2602_10431_amd as qt
    c = s["case"]
    return qt.qtale_paged_attention(s["kv"], 0, s["q"], s["offs"], first=s["first"], slots=s["slots"], out=s["out"], window=c["window"],
                                    sinks=c["sinks"], max_new=s["max_new"], max_len=s["max_len"], workspace=s["workspace"])


def _own_pages(s):
    import paper_2602_10431_amd as qt
    c, kv = s["case"], s["kv"]
    out = dict(table=s["table"], kv_len=s["kv_len"], kv_cap=s["kv_cap"], refs=s["refs"], bits=s["bits"])
    if c["kind"] == "branch":
        qt.qtale_pages_fork(kv, s["src"], s["dst"])
        qt.qtale_pages_reserve(kv, s["offs"], slots=s["slots"], first=s["first"], missing=s["missing"], workspace=s["workspace"])
        return dict(out, first=s["first"], missing=s["missing"], k=s["k"], v=s["v"])
    if c["kind"] == "compact":
        qt.qtale_pages_compact(kv, s["n_live"], workspace=s["workspace"])
        return dict(out, n_live=s["n_live"], k=s["k"], v=s["v"])
    qt.qtale_pages_release(kv, s["ended"])
    qt.qtale_pages_trim(kv, c["window"], c["sinks"], slots=s["going"])
    return out


def _rows(s):
    """Sequence of every new token and its place in the sequence's cache."""
    n = torch.diff(s["offs"].long())
    seq = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n, output_size=sum(s["new"]))
    at = s["first"].long()[seq] + torch.arange(seq.numel(), device="cuda") - s["offs"].long()[seq]
    return seq, at


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


def _plain_rope(s):
    c = s["case"]
    nh, nkv, d = SHAPES[c["shape"]]
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos, sin = ((f(angle).float() * s["magnitude"])[:, None] for f in (torch.cos, torch.sin))
    q, k, v = s["qkv"].split((nh, nkv, nkv), 1)
    s["out"].copy_(_turn(q.float(), cos, sin, c["layout"], _rotary(c)))
    seq, at = _rows(s)
    page = s["table"][0].long()[s["slots"].long()[seq], at // c["page"]]
    s["k"][page, :, at % c["page"]] = _turn(k.float(), cos, sin, c["layout"], _rotary(c)).to(s["k"].dtype)
    s["v"][page, :, at % c["page"]] = v
    return dict(q=s["out"], k=s["k"], v=s["v"])


def _plain_attend(s):
    c = s["case"]
    nh, nkv, d = SHAPES[c["shape"]]
    at = 0
    for b, (n, o) in enumerate(zip(s["new"], s["old"])):
        pages = s["table"][0, s["slots"][b].long(), : -(-(n + o) // c["page"])].long()
        gone = (pages < 0).repeat_interleave(c["page"])[: n + o]
        k, v = (t[pages.clamp(min=0)].transpose(0, 1).reshape(nkv, -1, d)[:, : n + o].float().masked_fill(gone[:, None], 0.0)
                for t in (s["k"], s["v"]))
        place, key = torch.arange(o, o + n, device="cuda")[:, None], torch.arange(n + o, device="cuda")
        seen = (key <= place) & ~gone
        if c["window"]:
            seen &= (key > place - c["window"]) | (key < c["sinks"])
        q = s["q"][at: at + n].float().view(n, nkv, nh // nkv, d).permute(1, 2, 0, 3).reshape(nkv, -1, d)
        score = torch.bmm(q, k.transpose(1, 2).contiguous()).view(nkv, nh // nkv, n, n + o) * d ** -0.5
        score = score.masked_fill_(~seen, float("-inf"))
        p = torch.exp_(score.sub_(score.amax(3, keepdim=True)))
        p = p.div_(p.sum(3, keepdim=True)).view(nkv, -1, n + o)
        s["out"][at: at + n] = torch.bmm(p, v).view(nkv, nh // nkv, n, d).permute(2, 0, 1, 3).reshape(n, nh, d).to(s["out"].dtype)
        at += n
    return s["out"]


def _plain_pages(s):
    c, page = s["case"], s["case"]["page"]
    table, kv_len, kv_cap, refs = s["table"], s["kv_len"], s["kv_cap"], s["refs"]
    out = dict(table=table, kv_len=kv_len, kv_cap=kv_cap, refs=refs, bits=s["bits"])
    place = torch.arange(table.shape[2], device="cuda")

    def count(entries, by):
        refs.index_add_(0, entries, torch.full_like(entries, by, dtype=torch.int32))

    if c["kind"] == "branch":
        src, dst, slots = s["src"].long(), s["dst"].long(), s["slots"].long()
        written = -(-kv_len[:, src] // page)
        rows = torch.where(place < written[..., None], table[:, src], -1)
        table[:, dst], kv_len[:, dst], kv_cap[:, dst] = rows, kv_len[:, src], written * page
        count(rows[rows >= 0].long(), 1)
        # room for the next tokens, in the order of layers and then sequences
        first, cap = kv_len[:, slots].clone(), kv_cap[:, slots]
        n = torch.diff(s["offs"])[None]
        last = table[:, slots].gather(2, (first // page).clamp(max=table.shape[2] - 1).long()[..., None])[..., 0]
        partial = (n > 0) & (first % page != 0) & (last >= 0)
        shared = refs[last.clamp(min=0).long()]
        same = (last[:, :, None] == last[:, None, :]) & partial[:, :, None] & partial[:, None, :]
        earlier = torch.ones(slots.numel(), slots.numel(), dtype=torch.bool, device="cuda").tril(-1)
        copied = partial & (shared - (same & earlier).sum(2) > 1)    # each of a page's holders but the last takes a copy
        wanted = torch.minimum(-(-(first + n) // page), torch.tensor(table.shape[2], device="cuda"))
        extra = torch.where(n > 0, (wanted - cap // page).clamp(min=0), 0)
        need = (copied + extra).flatten()
        start = need.cumsum(0) - need
        free = torch.nonzero(refs == 0)[:, 0]
        got = torch.minimum((free.numel() - start).clamp(min=0), need)
        start, got_all = start.view_as(first), got.view_as(first)
        copied = copied & (got_all > 0)
        if copied.any():
            lay, b = torch.nonzero(copied, as_tuple=True)
            new, old = free[start[lay, b]], last[lay, b].long()
            keep = torch.arange(page, device="cuda") < (first[lay, b] % page)[:, None]
            for t in (s["k"], s["v"]):
                t[new] = torch.where(keep[:, None, :, None], t[old], t[new])
            table[lay, slots[b], (first[lay, b] // page).long()] = new.int()
            count(old, -1)
            count(new, 1)
        granted = got_all - copied.int()
        j = torch.arange(int(extra.max()), device="cuda")
        lay, b, j = torch.nonzero(j < granted[..., None], as_tuple=True)
        new = free[start[lay, b] + copied[lay, b] + j]
        table[lay, slots[b], (cap[lay, b] // page).long() + j] = new.int()
        count(new, 1)
        kv_cap[:, slots] = cap + granted.int() * page
        copy_missed = (need.view_as(first) > extra) & (got_all == 0)  # a shared page that could not be copied takes no token
        kv_len[:, slots] = torch.where(copy_missed, first, torch.minimum(first + n, kv_cap[:, slots]))
        s["bits"].copy_(_words(refs == 0))
        return dict(out, first=first, missing=(need - got).sum().int().view(1), k=s["k"], v=s["v"])
    if c["kind"] == "compact":
        live = refs > 0
        n_live = int(live.sum())
        src, dst = torch.nonzero(live[n_live:])[:, 0] + n_live, torch.nonzero(~live[:n_live])[:, 0]
        for t in (s["k"], s["v"]):
            t[dst] = t[src]
        moved = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
        moved[src] = dst.int()
        table.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()], table))
        refs[dst] = refs[src]
        refs[src] = 0
        s["bits"].copy_(_words(refs == 0))
        return dict(out, n_live=live.sum().int().view(1), k=s["k"], v=s["v"])
    ended, going = s["ended"].long(), s["going"].long()
    rows = table[:, ended]
    count(rows[rows >= 0].long(), -1)
    table[:, ended], kv_len[:, ended], kv_cap[:, ended] = -1, 0, 0
    rows, n = table[:, going], kv_len[:, going, None]
    left = (rows >= 0) & ((place + 1) * page <= n + 1 - c["window"]) & (place * page >= c["sinks"])
    count(rows[left].long(), -1)
    table[:, going] = torch.where(left, -1, rows)
    s["bits"].copy_(_words(refs == 0))
    return out


# ---- the same results in 64 bits ------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] in ("branch", "compact", "retire"):
        return None                                               # whole numbers and copies
    nh, nkv, d = SHAPES[case["shape"]]
    dtype, page = TYPES[case["dtype"]], case["page"]
    s = _state(case, seed)
    table, slots = s["table"][0].tolist(), s["slots"].tolist()
    if case["kind"] == "rope":
        f, rd = s["freqs"], _rotary(case)
        angle = torch.outer(s["positions"].double(), f)
        turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)
        x = s["qkv"].double()
        head = x[:, : nh + nkv, :rd]
        pairs = head.reshape(-1, nh + nkv, rd // 2, 2) if case["layout"] == "interleaved" else head.reshape(-1, nh + nkv, 2, rd // 2).transpose(2, 3)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        x[:, : nh + nkv, :rd] = (z if case["layout"] == "interleaved" else z.transpose(2, 3)).reshape(-1, nh + nkv, rd)
        k, v = s["k"].double(), s["v"].double()
        t = 0
        for b, (n, o) in enumerate(zip(s["new"], s["old"])):
            for j in range(o // page, -(-(o + n) // page)):       # page by page
                lo, hi = max(o, j * page), min(o + n, (j + 1) * page)
                rows = x[t + lo - o: t + hi - o].transpose(0, 1)
                p = table[slots[b]][j]
                k[p, :, lo - j * page: hi - j * page], v[p, :, lo - j * page: hi - j * page] = rows[nh: nh + nkv], rows[nh + nkv:]
            t += n
        return dict(q=x[:, :nh].contiguous(), k=k, v=v)
    out = torch.empty(sum(s["new"]), nh, d, dtype=torch.float64, device="cuda")
    t = 0
    for b, (n, o) in enumerate(zip(s["new"], s["old"])):
        at = [(j * page, table[slots[b]][j]) for j in range(-(-(o + n) // page)) if table[slots[b]][j] >= 0]
        where = torch.cat([torch.arange(a, min(a + page, o + n)) for a, _ in at]).cuda()
        ids = torch.tensor([p for _, p in at], device="cuda")
        token = torch.cat([torch.arange(i * page, i * page + min(page, o + n - a)) for i, (a, _) in enumerate(at)]).cuda()
        for h in range(nkv):
            kh, vh = (x[ids, h].reshape(-1, d)[token].double() for x in (s["k"], s["v"]))
            for i in range(h * (nh // nkv), (h + 1) * (nh // nkv)):
                z = (s["q"][t: t + n, i].double() @ kh.t()) / math.sqrt(d)
                back = torch.arange(o, o + n, device="cuda")[:, None] - where[None]
                hidden = back < 0
                if case["window"]:
                    hidden |= (back >= case["window"]) & (where >= case["sinks"])[None]
                out[t: t + n, i] = torch.softmax(z.masked_fill(hidden, -math.inf), 1) @ vh
        t += n
    return out
