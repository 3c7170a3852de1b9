"""Performance cases of the operators around a 16-bit key/value cache and the verification of drafts by sampling, through the library's public Python entry points.

The cache holds keys and values in bf16 or f16, in pages as the library documents them:

  pages  [page][kv head][K | V][page_tokens / 16][16 * head_dim]   in a block of 16 tokens:
         K  [head_dim / 8][token][8 features]
         V  [head_dim / 32][token / 4][feature % 16][feature / 16 % 2][token % 4]

rotate  rotary positions of rows of heads: pairs of features half a rotated part apart or next to each other, all of the head or a part of it, frequencies as they are
        or scaled for long contexts
append  writes new tokens' keys, rotated on the way, and values into the pages, and rotates the queries of the same rows
attend  attention of blocks of rows (decoded tokens, draft trees, prompts) over such a cache: a row sees the prefix and, of its own block, the rows up to its own or
        (draft tree, of any number of nodes) those that its mask names
verify  drafted tokens accepted or not against the target's probabilities, from given random numbers, and the token that follows: chains drawn from a drafter's
        probabilities, trees of given tokens; with the target's probability of each
keep    after a tree: the accepted path's keys and values moved behind the prefix

All take ragged batches: row_start [sequences + 1], prefix_len [sequences], page_table [sequences][pages], on the GPU.
"""
import math
import random

import torch

from pv_inputs import CONFIGS

own = False

PAGE = 16                                   # tokens a page, as in the repository's configurations
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
WIDTHS = ("1b", "7b", "8b", "70b")
# frequencies for contexts longer than the trained one: all divided; divided where a feature makes few turns in the trained context, kept where it makes many, by the
# number of turns or by the feature's place in between
SCALINGS = {"none": None, "linear": {"kind": "linear", "factor": 4.0}, "turns": {"kind": "turns", "factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192},
            "ramp": {"kind": "ramp", "factor": 16.0, "slow": 1.0, "fast": 32.0, "original": 4096}}


def listed():
    return [
        # the smallest call: the queries of one decoded token
        {"name": "rotate_8b_1", "do": "rotate", "heads": 32, "head_dim": 128, "part": 128, "dtype": "bf16", "rows": 1, "far": 5000, "interleaved": False, "scaling": "none"},
        # a prompt's queries and keys in 32 bits, half of each head rotated, neighbours as pairs, positions of a long context
        {"name": "rotate_half_8191", "do": "rotate", "heads": 40, "head_dim": 128, "part": 64, "dtype": "f32", "rows": 8191, "far": 120000, "interleaved": True, "scaling": "turns"},
        # a decoding step: one token of each of 64 sequences, drafter's shape
        {"name": "append_1b_64x1", "do": "append", "width": "1b", "dtype": "bf16", "seqs": 64, "prefix": 2048, "rows": 1, "interleaved": False, "scaling": "turns"},
        # prompts of four sequences, the final stage's shape
        {"name": "append_70b_4x4096", "do": "append", "width": "70b", "dtype": "bf16", "seqs": 4, "prefix": 37, "rows": 4096, "interleaved": False, "scaling": "none"},
        # a decoding batch of 32 sequences of different lengths
        {"name": "attend_8b_32x1", "do": "attend", "width": "8b", "dtype": "bf16", "seqs": 32, "prefix": 8192, "rows": 1},
        # a draft tree of 200 nodes over an odd context
        {"name": "attend_70b_tree_200", "do": "attend", "width": "70b", "dtype": "f16", "seqs": 1, "prefix": 4101, "rows": 200, "tree": True},
        # two long prompts put in on top of a context: the largest
        {"name": "attend_8b_2x2048", "do": "attend", "width": "8b", "dtype": "bf16", "seqs": 2, "prefix": 6100, "rows": 2048},
        # one sequence's window of eight drafts: latency counts
        {"name": "verify_8b_1x8", "do": "verify", "vocab": 128256, "dtype": "f32", "seqs": 1, "rows": 9},
        # a serving step: up to five drafts of each of 64 sequences, among them some that want the most probable token
        {"name": "verify_7b_64x5", "do": "verify", "vocab": 32000, "dtype": "bf16", "seqs": 64, "rows": 6, "greedy": True},
        # draft trees of up to 48 nodes of 16 sequences
        {"name": "verify_8b_tree_16x48", "do": "verify", "vocab": 128256, "dtype": "bf16", "seqs": 16, "rows": 48, "tree": True},
        # one accepted path of a small tree
        {"name": "keep_8b_1", "do": "keep", "width": "8b", "dtype": "bf16", "seqs": 1, "prefix": 301, "rows": 24},
        # paths of 32 larger ones
        {"name": "keep_70b_32", "do": "keep", "width": "70b", "dtype": "f16", "seqs": 32, "prefix": 300, "rows": 96},
    ]


def draw(rng):
    """One more case: any operator, any width, one to 64 sequences, prefixes of none to 60000 tokens, one to 16384 rows, trees of 2 to 500 nodes, vocabularies of 50 to 200000 tokens."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    do = rng.choice(["rotate", "append", "attend", "attend", "attend", "verify", "verify", "keep"])
    while True:
        case = {"do": do, "dtype": rng.choice(["bf16", "f16"]), "seqs": rng.choice([1, log(1, 64)])}
        if do in ("rotate", "append"):
            case.update(interleaved=rng.random() < 0.4, scaling=rng.choice(list(SCALINGS)))
        if do in ("append", "attend", "keep"):
            case["width"] = rng.choice(WIDTHS)
        if do == "rotate":
            del case["seqs"]
            hd = rng.choice([64, 96, 128, 256])
            case.update(heads=log(1, 72), head_dim=hd, part=rng.choice([hd, hd, 16 * rng.randint(1, hd // 16)]), dtype=rng.choice(["bf16", "f16", "f32"]), rows=log(1, 16384), far=log(10, 1000000))
        elif do == "append":
            case.update(rows=log(1, 8192), prefix=log(1, 60001) - 1)
            if rng.random() < 0.2:
                case["dtype"] = "f32"
        elif do == "attend":
            kind = rng.choice(["decode", "tree", "prompt"])
            case.update(rows=1 if kind == "decode" else log(2, 500) if kind == "tree" else log(2, 2048), prefix=log(1, 60001) - 1)
            if kind == "tree":
                case["tree"] = True
        elif do == "verify":
            case.update(vocab=rng.choice([1024, 32000, 128256, log(50, 200000)]), dtype=rng.choice(["bf16", "f16", "f32"]), rows=log(1, 17))
            if rng.random() < 0.4:
                case.update(tree=True, rows=log(2, 128))
            if rng.random() < 0.3:
                case["greedy"] = True
        else:
            case.update(rows=log(2, 256), prefix=log(1, 2000) - 1)
        w = work(case)
        if w["bytes"] > 6e8 or w["flops"] > 3.3e11 or (do == "verify" and case["seqs"] * case["rows"] * case["vocab"] > 1.0e8):
            continue
        if do in ("append", "attend", "keep") and case["seqs"] * (case["prefix"] + case["rows"]) > 300000:
            continue
        return case


# ---- the sequences of a case ----

def lengths(case):
    """(prefix, rows) of every sequence: ragged from the largest down, and in larger batches one without rows."""
    n = case["seqs"]
    rows = [max(1, case["rows"] - (case["rows"] * i) // (2 * n)) for i in range(n)]
    prefix = [max(0, case.get("prefix", 0) * (n - i) // n - 3 * i) for i in range(n)]
    if n >= 8:
        rows[n // 2] = 0
    return prefix, rows


def tables(case, g):
    prefix, rows = lengths(case)
    pages = -(-max(p + r for p, r in zip(prefix, rows)) // PAGE)
    table = torch.randperm(pages * case["seqs"], generator=g, device="cuda").to(torch.int32).view(case["seqs"], pages)
    return torch.tensor(prefix, dtype=torch.int32, device="cuda"), starts(rows), table


def starts(rows):
    return torch.tensor([0] + rows).cumsum(0).to(torch.int32).cuda()


def parents_of(n, r, width):
    """A tree's nodes: 0 is its root, every other one hangs under one of the few before it."""
    return [-1] + [r.randint(max(0, (i - 1) // width - 2), (i - 1) // width) for i in range(1, n)]


def tree_masks(case, seed):
    """For every row of a tree its ancestors and itself: [rows, words], bit t of word w names row 64 w + t of the sequence."""
    r, words, out = random.Random(seed), -(-case["rows"] // 64), []
    for n in lengths(case)[1]:
        mine = []
        for i, up in enumerate(parents_of(n, r, 3) if n else []):
            mine.append((1 << i) | (mine[up] if up >= 0 else 0))
        for m in mine:
            w = [(m >> (64 * k)) & ((1 << 64) - 1) for k in range(words)]
            out.append([x - (1 << 64) if x >> 63 else x for x in w])
    return torch.tensor(out, dtype=torch.int64).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = DTYPES[case["dtype"]]
    if case["do"] == "rotate":
        state = {"do": "rotate", "case": case, "x": torch.randn(case["rows"], case["heads"], case["head_dim"], generator=g, device="cuda").to(t),
                 "positions": torch.randint(0, case["far"], (case["rows"],), generator=g, device="cuda", dtype=torch.int32)}
        if own:
            import paper_2505_01572_amd as pv
            state["rotary"] = pv.Rotary(case["head_dim"], rotary_dim=case["part"], base=500000.0, interleaved=case["interleaved"], scaling=SCALINGS[case["scaling"]])
        return state
    if case["do"] == "verify":
        return prepare_verify(case, seed, g)
    s = CONFIGS[case["width"]]
    prefix, start, table = tables(case, g)
    total, n = sum(lengths(case)[1]), table.numel()
    kept = torch.bfloat16 if case["dtype"] == "f32" else t
    pages = torch.randn(n, s.n_kv_heads, 2, PAGE * s.head_dim, generator=g, device="cuda", dtype=torch.float32 if n < 20000 else kept).to(kept)      # a used cache
    state = {"do": case["do"], "case": case, "pages": pages, "prefix": prefix, "start": start, "table": table, "rows": total}
    if own:
        import paper_2505_01572_amd as pv
        state["pool"] = pv.KV16Pool(n, s.n_kv_heads, s.head_dim, PAGE, dtype=kept, pages=pages)
        state["seqs"] = pv.KVSeqs(start, prefix, table)
    if case["do"] == "append":                                                   # parts of one row of a fused projection, as a decoder has them
        qkv = torch.randn(total, s.n_q_heads + 2 * s.n_kv_heads, s.head_dim, generator=g, device="cuda").to(t)
        state["q"], state["k"], state["v"] = qkv[:, : s.n_q_heads], qkv[:, s.n_q_heads: s.n_q_heads + s.n_kv_heads], qkv[:, s.n_q_heads + s.n_kv_heads:]
        if own:
            state["rotary"] = pv.Rotary(s.head_dim, base=s.rope_base, interleaved=case["interleaved"], scaling=SCALINGS[case["scaling"]])
    elif case["do"] == "attend":
        state["q"] = (torch.randn(total, s.n_q_heads, s.head_dim, generator=g, device="cuda") * 1.5).to(t)
        state["mask"] = tree_masks(case, seed) if case.get("tree") else None
    else:                                                                        # paths of a few nodes, of numbers past the path's own length
        r, path, accepted = random.Random(seed), [], []
        for rows in lengths(case)[1]:
            a = r.randint(0, min(8, (rows - 1) // 2)) if rows else 0
            path += ([0] + sorted(r.sample(range(a + 1, rows), a)) + [-1] * (rows - 1 - a)) if rows else []
            accepted.append(a)
        state["path"], state["accepted"] = torch.tensor(path, dtype=torch.int32).cuda(), torch.tensor(accepted, dtype=torch.int32).cuda()
    return state


def prepare_verify(case, seed, g):
    """Logits of a step's rows, and drafts: drawn from a drafter that is near the target (chains), or the tokens it finds most probable (trees)."""
    rows, vocab, r = lengths(case)[1], case["vocab"], random.Random(seed)
    total, n = sum(rows), case["seqs"]
    logits = torch.randn(total, vocab, generator=g, device="cuda") * 2.5
    logits[:, : max(1, vocab // 50)].mul_(2.0)                                   # some tokens stand out, as in a trained model
    near = logits + torch.randn(total, vocab, generator=g, device="cuda") * 0.5
    temperature = torch.tensor([0.0 if case.get("greedy") and i % 4 == 3 else 0.6 + 0.1 * (i % 5) for i in range(n)], device="cuda")
    state = {"do": "verify", "case": case, "logits": logits.to(DTYPES[case["dtype"]]), "start": starts(rows), "temperature": temperature,
             "u": torch.rand(total, 2, generator=g, device="cuda"), "probs": None, "parent": None, "rows": total, "most": max(rows)}
    if case.get("tree"):
        parent = [p for m in rows for p in (parents_of(m, r, 3) if m else [])]
        up, rank = torch.tensor(parent), []
        row0 = [sum(rows[:i]) for i, m in enumerate(rows) for _ in range(m)]
        count = {}
        for i, p in enumerate(parent):                                           # a node's children carry its first, second ... token
            rank.append(count.get((row0[i], p), 0))
            count[(row0[i], p)] = rank[-1] + 1
        best = near.topk(min(vocab, max(rank) + 1), 1).indices
        at = (torch.tensor(row0) + up.clamp(min=0)).cuda()
        state["tokens"] = best[at, torch.tensor(rank).cuda()].to(torch.int32)
        state["parent"] = up.to(torch.int32).cuda()
    else:                                                                        # row j: drawn from what the drafter made of the row before it
        q = torch.softmax(near / temperature.repeat_interleave(torch.tensor(rows).cuda()).clamp(min=0.3)[:, None], 1).roll(1, 0)
        state["tokens"] = torch.multinomial(q, 1, generator=g)[:, 0].to(torch.int32)
        state["probs"] = q
    return state


# ---- the plain forms ----

def frequencies(base, part, scaling):
    """Radians a position of every pair, in 64 bits, and what the rotated numbers are multiplied by."""
    i = torch.arange(part // 2, dtype=torch.float64, device="cuda")
    f = base ** (-2 * i / part)
    if scaling is None:
        return f, 1.0
    if scaling["kind"] == "linear":
        return f / scaling["factor"], 1.0
    if scaling["kind"] == "turns":
        turns = scaling["original"] * f / (2 * math.pi)
        keep = ((turns - scaling["low"]) / (scaling["high"] - scaling["low"])).clamp(0, 1)
        return keep * f + (1 - keep) * f / scaling["factor"], 1.0
    place = lambda turns: part * math.log(scaling["original"] / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    first, last = max(math.floor(place(scaling["fast"])), 0), min(math.ceil(place(scaling["slow"])), part - 1)
    keep = 1 - ((i - first) / max(last - first, 0.001)).clamp(0, 1)
    return keep * f + (1 - keep) * f / scaling["factor"], 0.1 * math.log(scaling["factor"]) + 1


def rotated(x, positions, base, part, interleaved, scaling):
    """Rows of heads turned by their positions, in 32 bits."""
    f, much = frequencies(base, part, scaling)
    angle = positions.double()[:, None] * f
    c, s = (much * torch.cos(angle)).float()[:, None], (much * torch.sin(angle)).float()[:, None]
    x = x.float()
    a, b = (x[..., 0:part:2], x[..., 1:part:2]) if interleaved else (x[..., : part // 2], x[..., part // 2: part])
    y = torch.stack([a * c - b * s, a * s + b * c], -1 if interleaved else -2).flatten(-2)
    return torch.cat([y, x[..., part:]], -1)


def plain_rotate(state):
    c, x = state["case"], state["x"]
    return {"out": rotated(x, state["positions"], 500000.0, c["part"], c["interleaved"], SCALINGS[c["scaling"]]).to(x.dtype)}


def places(state):
    """Sequence, position, page and block within it of every row."""
    row = torch.arange(state["rows"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(state["start"], row, right=True) - 1
    pos = (state["prefix"][seq] + row - state["start"][seq]).long()
    return seq, pos, state["table"][seq, pos // PAGE].long(), pos % PAGE // 16


def views(pages):
    """The pool's keys and values, a dimension for each part of the layout."""
    n, h, _, size = pages.shape
    return pages.view(n, h, 2, PAGE // 16, size // PAGE // 8, 16, 8), pages.view(n, h, 2, PAGE // 16, size // PAGE // 32, 4, 16, 2, 4)


def put(pages, page, sub, off, k, v):
    kc, vc = views(pages)
    r, h, hd = k.shape
    kc[page, :, 0, sub, :, off] = k.to(pages.dtype).reshape(r, h, hd // 8, 8)
    vc[page, :, 1, sub, :, off // 4, :, :, off % 4] = v.to(pages.dtype).reshape(r, h, hd // 32, 2, 16).transpose(3, 4)


def gathered(pages, page, sub, off):
    """Keys and values of tokens, by their places: [...][head][feature] each."""
    kc, vc = views(pages)
    h, hd, lead = kc.shape[1], kc.shape[4] * 8, page.shape
    page, sub, off = page.reshape(-1), sub.reshape(-1), off.reshape(-1)
    k = kc[page, :, 0, sub, :, off].reshape(*lead, h, hd)
    v = vc[page, :, 1, sub, :, off // 4, :, :, off % 4].transpose(3, 4).reshape(*lead, h, hd)
    return k, v


def plain_append(state):
    c, s = state["case"], CONFIGS[state["case"]["width"]]
    _, pos, page, sub = places(state)
    turn = (pos, s.rope_base, s.head_dim, c["interleaved"], SCALINGS[c["scaling"]])
    put(state["pages"], page, sub, pos % 16, rotated(state["k"], *turn), state["v"].float())
    return {"pages": state["pages"], "q": rotated(state["q"], *turn).to(state["q"].dtype)}


def plain_attend(state):
    seq, pos, _, _ = places(state)
    q, start, prefix, table = state["q"], state["start"].long(), state["prefix"].long(), state["table"]
    n, keys = table.shape[0], table.shape[1] * PAGE
    at = torch.arange(keys, device="cuda")
    page = table.long()[:, at // PAGE]
    k, v = gathered(state["pages"], page, (at % PAGE // 16).expand(n, -1), (at % 16).expand(n, -1))
    h, hd = k.shape[2:]
    group, most = q.shape[1] // h, state["case"]["rows"]
    local = torch.arange(state["rows"], device="cuda") - start[seq]
    pad = torch.zeros(n, most, q.shape[1], hd, device="cuda")
    pad[seq, local] = q.float()
    see = torch.zeros(n, most, keys, dtype=torch.bool, device="cuda")
    slot = at[None] - prefix[seq][:, None]                                       # [row][key]: its slot in the sequence's block
    if state["mask"] is None:
        see[seq, local] = slot <= local[:, None]
    else:
        bits = ((state["mask"][:, :, None] >> torch.arange(64, device="cuda")) & 1).bool().flatten(1)
        inside = slot < torch.minimum(start[seq + 1] - start[seq], torch.tensor(bits.shape[1], device="cuda"))[:, None]
        see[seq, local] = (slot < 0) | (inside & bits.gather(1, slot.clamp(0, bits.shape[1] - 1)))
    del slot
    rows = pad.view(n, most, h, group, hd).permute(0, 2, 1, 3, 4).reshape(n * h, most * group, hd)
    s = rows @ k.float().permute(0, 2, 3, 1).reshape(n * h, hd, keys).contiguous()
    s = s.mul_(1 / math.sqrt(hd)).view(n, h, most, group, keys).masked_fill_(~see[:, None, :, None], -math.inf)
    top = s.amax(4, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(4, keepdim=True)
    out = p.view(n * h, most * group, keys) @ v.float().permute(0, 2, 1, 3).reshape(n * h, keys, hd).contiguous()
    out = out.view(n, h, most, group, hd) / torch.where(total == 0, 1.0, total)
    out = out.permute(0, 2, 1, 3, 4).reshape(n, most, h * group, hd)[seq, local]
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(n, most, h * group)[seq, local]
    return {"out": out.to(q.dtype), "lse": lse}


def plain_verify(state):
    """In 64 bits throughout: a token is drawn where a sum of many probabilities passes a random number."""
    start, n, total, vocab = state["start"].long(), state["start"].numel() - 1, state["rows"], state["logits"].shape[1]
    row = torch.arange(total, device="cuda")
    seq = torch.searchsorted(start, row, right=True) - 1
    local, count = row - start[seq], start[1:] - start[:-1]
    x, hot = state["logits"].double(), state["temperature"].double()
    p = torch.softmax(x / torch.where(hot > 0, hot, 1.0)[seq][:, None], 1)
    first = (x == x.amax(1, keepdim=True)).to(torch.int8).argmax(1)              # the lowest of the largest ones
    one = torch.zeros_like(p).scatter_(1, first[:, None], 1.0)
    p = torch.where((hot == 0)[seq][:, None], one, p)
    del x, one
    token, u = state["tokens"].long(), state["u"].double()
    ids = torch.arange(vocab, device="cuda")
    at0 = start[:-1].clamp(max=total - 1)
    up = (row - 1).clamp(min=0) if state["parent"] is None else start[seq] + state["parent"].long().clamp(min=0)
    above = p[up, token]
    probs = torch.where(local > 0, above, 1.0)
    if state["parent"] is None:
        ok = u[:, 0] * state["probs"].double().gather(1, token[:, None])[:, 0] < above
        stop = torch.where((local > 0) & ~ok, local - 1, count[seq] - 1)
        accepted = torch.full((n,), total, device="cuda").scatter_reduce(0, seq, stop, "amin")
        accepted = torch.where(count > 0, accepted, 0)
        here = (at0 + accepted).clamp(max=total - 1)
        left = p[here]
        rejected = accepted < count - 1
        rest = (left - state["probs"].double()[(here + 1).clamp(max=total - 1)]).clamp(min=0)
        left = torch.where((rejected & (rest.sum(1) > 0))[:, None], rest, left)
        path = None
    else:
        parent = state["parent"].long()
        node, depth = torch.zeros(n, dtype=torch.long, device="cuda"), torch.zeros(n, dtype=torch.long, device="cuda")
        path = torch.full((total + 1,), -1, dtype=torch.long, device="cuda")
        path[torch.where(count > 0, at0, total)] = 0
        left = p[at0]
        for i in range(1, state["most"]):                                        # a node's children come behind it, in the order they are tried in
            here = (at0 + i).clamp(max=total - 1)
            tried = (i < count) & (parent[here] == node)
            mine = left.gather(1, token[here][:, None])[:, 0]
            taken = tried & (u[here, 0] * left.sum(1) < mine)
            node = torch.where(taken, i, node)
            depth = depth + taken
            path[torch.where(taken, at0 + depth, total)] = i
            left = torch.where((tried & ~taken)[:, None] & (ids == token[here][:, None]), 0.0, left)
            left = torch.where(taken[:, None], p[here], left)
        accepted, path = depth, path[:total].to(torch.int32)
        here = (at0 + node).clamp(max=total - 1)
    sums = left.cumsum(1)
    passed = sums > u[here, 1][:, None] * sums[:, -1:]
    drawn = passed.to(torch.int8).argmax(1)
    out = {"accepted": accepted.to(torch.int32), "next_token": torch.where(count > 0, drawn, -1).to(torch.int32), "probs": probs.float()}
    if path is not None:
        out["path"] = path
    return out


def plain_keep(state):
    seq, pos, page, sub = places(state)
    local = torch.arange(state["rows"], device="cuda") - state["start"].long()[seq]
    source = torch.where(local <= state["accepted"].long()[seq], state["path"].long(), local)      # others stay
    source = state["prefix"].long()[seq] + source
    k, v = gathered(state["pages"], state["table"][seq, source // PAGE].long(), source % PAGE // 16, source % 16)
    put(state["pages"], page, sub, pos % 16, k, v)
    return {"pages": state["pages"]}


def run(state):
    if own:
        if state["do"] == "rotate":
            return {"out": state["rotary"].rotate(state["x"], state["positions"])}
        if state["do"] == "append":
            return {"pages": state["pages"], "q": state["pool"].append(state["seqs"], state["k"], state["v"], rotary=state["rotary"], q=state["q"])}
        if state["do"] == "attend":
            out, lse = state["pool"].attention(state["seqs"], state["q"], mask=state["mask"], return_lse=True)
            return {"out": out, "lse": lse}
        if state["do"] == "keep":
            state["pool"].keep(state["seqs"], state["path"], state["accepted"])
            return {"pages": state["pages"]}
        import paper_2505_01572_amd as pv
        got = pv.verify_drafts(state["start"], state["logits"], state["tokens"], state["u"], draft_probs=state["probs"], parent=state["parent"], temperature=state["temperature"])
        out = {"accepted": got.accepted, "next_token": got.next_token, "probs": got.probs}
        if state["parent"] is not None:
            out["path"] = got.path
        return out
    return {"rotate": plain_rotate, "append": plain_append, "attend": plain_attend, "verify": plain_verify, "keep": plain_keep}[state["do"]](state)


# ---- what a pass cannot do without ----

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    if case["do"] == "rotate":
        n = case["rows"] * case["heads"]
        return {"bytes": float(n * case["head_dim"] * 2 * size + 4 * case["rows"]), "flops": 3.0 * n * case["part"]}
    prefix, rows = lengths(case)
    if case["do"] == "verify":                                                   # every row of logits, of the drafter's probabilities one a sequence
        n = sum(rows) * case["vocab"]
        return {"bytes": float(n * size + (0 if case.get("tree") else 4 * case["seqs"] * case["vocab"]) + 24 * sum(rows)), "flops": 4.0 * n}
    s = CONFIGS[case["width"]]
    token = 2 * s.n_kv_heads * s.head_dim                                        # elements of one token's keys and values
    if case["do"] == "append":
        q = s.n_q_heads * s.head_dim
        return {"bytes": float(sum(rows) * (token * (size + 2) + 2 * q * size)), "flops": 3.0 * sum(rows) * (token / 2 + q)}
    if case["do"] == "keep":
        moved = max(1.0, sum(min(8, max(0, r - 1) // 2) for r in rows) / 2)      # (in the mean)
        return {"bytes": moved * token * 2 * size, "flops": moved * token}
    keys = sum(p + r for p, r in zip(prefix, rows) if r)
    pairs = sum(r * p + (r * (r + 1) / 2) for p, r in zip(prefix, rows))
    return {"bytes": float(keys * token * size + sum(rows) * s.n_q_heads * (2 * s.head_dim * size + 4)), "flops": 4.0 * pairs * s.n_q_heads * s.head_dim}


# ---- the same in 64 bits, sequence by sequence ----

def exact_turn(x, positions, base, part, interleaved, scaling):
    """Pairs of features as complex numbers, times one of the position's angle."""
    i = torch.arange(0, part, 2, dtype=torch.float64, device="cuda")
    f, much = torch.exp(-i / part * math.log(base)), 1.0
    if scaling is not None:
        if scaling["kind"] == "linear":
            share = torch.zeros_like(f)                                          # how much of the frequency stays as it is
        elif scaling["kind"] == "turns":
            share = torch.clamp((f * scaling["original"] / math.tau - scaling["low"]) / (scaling["high"] - scaling["low"]), 0.0, 1.0)
        else:
            where = [part / 2 * math.log(scaling["original"] / math.tau / t, base) for t in (scaling["fast"], scaling["slow"])]
            lo, hi = max(0, math.floor(where[0])), min(part - 1, math.ceil(where[1]))
            share = 1.0 - torch.clamp((i / 2 - lo) / max(hi - lo, 0.001), 0.0, 1.0)
            much = 1.0 + math.log(scaling["factor"]) / 10
        f = f * (share + (1.0 - share) / scaling["factor"])
    turn = torch.polar(torch.full_like(f, much).expand(len(positions), -1).contiguous(), positions.double()[:, None] * f)[:, None]
    y = x.double().clone()
    first, second = (slice(0, part, 2), slice(1, part, 2)) if interleaved else (slice(0, part // 2), slice(part // 2, part))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def spots(table, pos, hd, which):
    """Page and place within a head's keys or values of every feature of a sequence's tokens."""
    e, off, sub = torch.arange(hd, device="cuda")[None], pos[:, None] % 16, pos[:, None] % PAGE // 16
    if which == 0:
        at = e // 8 * 128 + off * 8 + e % 8
    else:
        at = e // 32 * 512 + off // 4 * 128 + e % 16 * 8 + e // 16 % 2 * 4 + off % 4
    return table.long()[pos // PAGE], sub * 16 * hd + at


def exact(case, seed):
    state = prepare(case, seed)
    if case["do"] == "rotate":
        return {"out": exact_turn(state["x"], state["positions"], 500000.0, case["part"], case["interleaved"], SCALINGS[case["scaling"]])}
    if case["do"] == "verify":
        return exact_verify(case, state)
    s, table = CONFIGS[case["width"]], state["table"]
    prefix, rows = lengths(case)
    heads = torch.arange(s.n_kv_heads, device="cuda")[None, :, None]
    if case["do"] in ("append", "keep"):
        pages, r0, q = state["pages"].double(), 0, []
        for i, (p, r) in enumerate(zip(prefix, rows)):
            pos = torch.arange(p, p + r, device="cuda")
            if case["do"] == "append":
                turn = (pos, s.rope_base, s.head_dim, case["interleaved"], SCALINGS[case["scaling"]])
                q.append(exact_turn(state["q"][r0:r0 + r], *turn))
                new = exact_turn(state["k"][r0:r0 + r], *turn), state["v"][r0:r0 + r].double()
            elif r:
                n = int(state["accepted"][i]) + 1
                pos, came = pos[:n], p + state["path"][r0:r0 + n].long()
                new = []
                for which in (0, 1):
                    page, at = spots(table[i], came, s.head_dim, which)
                    new.append(pages[page[:, None, None], heads, which, at[:, None, :]])
            for which in (0, 1) if r else ():
                page, at = spots(table[i], pos, s.head_dim, which)
                pages[page[:, None, None], heads, which, at[:, None, :]] = new[which]
            r0 += r
        return {"pages": pages, "q": torch.cat(q)} if case["do"] == "append" else {"pages": pages}
    if work(case)["flops"] > 2e12:
        return None
    outs, lses, r0, group = [], [], 0, s.n_q_heads // s.n_kv_heads
    for i, (p, r) in enumerate(zip(prefix, rows)):
        if r == 0:
            continue
        pos = torch.arange(p + r, device="cuda")
        kv = []
        for which in (0, 1):
            page, at = spots(table[i], pos, s.head_dim, which)
            kv.append(state["pages"][page[:, None, None], heads, which, at[:, None, :]].double())
        if case.get("tree"):
            t = torch.arange(r, device="cuda")
            bits = (state["mask"][r0:r0 + r][:, t // 64] >> (t % 64)) & 1
            see = torch.cat([torch.ones(r, p, dtype=torch.bool, device="cuda"), bits.bool()], 1)
        else:
            see = pos[None] <= p + torch.arange(r, device="cuda")[:, None]
        out = torch.empty(r, s.n_q_heads, s.head_dim, dtype=torch.float64, device="cuda")
        lse = torch.empty(r, s.n_q_heads, dtype=torch.float64, device="cuda")
        for head in range(s.n_q_heads):
            sc = state["q"][r0:r0 + r, head].double() @ kv[0][:, head // group].t() / math.sqrt(s.head_dim)
            sc = sc.masked_fill(~see, -math.inf)
            lse[:, head] = torch.logsumexp(sc, 1)
            out[:, head] = torch.softmax(sc, 1) @ kv[1][:, head // group]
        outs.append(out)
        lses.append(lse)
        r0 += r
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def exact_verify(case, state):
    """Draft by draft, with the probabilities that are left made to sum to one again after each refusal."""
    rows, accepted, following, path, probs, r0 = lengths(case)[1], [], [], [], [], 0
    tokens, u, temperature = state["tokens"].tolist(), state["u"].double().tolist(), state["temperature"].tolist()
    parent = state["parent"].tolist() if state["parent"] is not None else None

    def target(row, t):
        x = state["logits"][row].double()
        if t == 0:
            p = torch.zeros_like(x)
            p[int((x == x.max()).nonzero()[0])] = 1.0
            return p
        e = torch.exp((x - x.max()) / t)
        return e / e.sum()

    for i, r in enumerate(rows):
        went, node, p = [0], 0, target(r0, temperature[i]) if r else None
        if r:
            probs.append(torch.ones((), dtype=torch.float64, device="cuda"))
        for j in range(1, r):
            up = parent[r0 + j] if parent is not None else j - 1
            probs.append(target(r0 + up, temperature[i])[tokens[r0 + j]])
            if up != node:
                continue
            t = tokens[r0 + j]
            q = state["probs"][r0 + j].double() if parent is None else None
            if u[r0 + j][0] * (1.0 if q is None else float(q[t])) < float(p[t]):
                node, p = j, target(r0 + j, temperature[i])
                went.append(j)
            elif q is None:
                p = p.clone()
                p[t] = 0.0
                p = p / p.sum()
            else:
                rest = torch.relu(p - q)
                p = rest / rest.sum() if float(rest.sum()) > 0 else p
        accepted.append(len(went) - 1 if r else 0)
        if r:
            reach = torch.cumsum(p, 0)
            following.append(int((reach > u[r0 + node][1] * reach[-1]).nonzero()[0]))
            path += went + [-1] * (r - len(went))
        else:
            following.append(-1)
        r0 += r
    out = {"accepted": torch.tensor(accepted, dtype=torch.int32, device="cuda"), "next_token": torch.tensor(following, dtype=torch.int32, device="cuda"), "probs": torch.stack(probs)}
    if parent is not None:
        out["path"] = torch.tensor(path, dtype=torch.int32, device="cuda")
    return out
