"""The operators of a step of several tokens, as timed cases.

Five operators:

* ``prompt``: prompts, or chunks of prompts, attend to the paged cache and to
  themselves, with capped scores, a bias by distance, windows, prefixes and
  documents (dsim_prompt_attention).
* ``tree``: a tree of drafted tokens attends to the cache and to each token's
  own ancestors (dsim_tree_attention).
* ``axes``: new keys and values are rotated by positions on several axes and
  written into the cache at places of their own (dsim_kv_append_axes).
* ``fork``: a step of a search: the losers' pages are released, the winners
  forked into their rows, room for the next token reserved (dsim_kv_release,
  dsim_kv_fork, dsim_kv_reserve).
* ``compact``: kept tokens of a sequence move to its front
  (dsim_kv_compact).

``run`` computes them from elementary torch operations, or, where ``own`` is
true, calls the framework's operators.  Lengths of a ragged batch are spread
evenly over the case's range and dealt out by the seed, so that a case's work
does not depend on the seed.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2, "e4m3": 1}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _prompt(name, b, lo, hi, heads, kv_heads, d, dtype, cache, page, past=0, window=0, cap=0.0, slopes=False, prefix=0,
            docs=0, scales=False):
    """b sequences with lo..hi new tokens each behind `past` cached ones.
    prefix: the first 1/prefix of a sequence is seen by all of it; docs: a
    sequence is that many documents end to end."""
    return {"name": name, "op": "prompt", "b": b, "lo": lo, "hi": hi, "heads": heads, "kv_heads": kv_heads, "d": d,
            "dtype": dtype, "cache": cache, "page": page, "past": past, "window": window, "cap": cap,
            "slopes": slopes, "prefix": prefix, "docs": docs, "scales": scales}


def _tree(name, b, lo, hi, nodes, heads, kv_heads, d, dtype, cache, page, window=0, cap=0.0, slopes=False,
          scales=False, ragged=False):
    """b sequences of lo..hi cached tokens with `nodes` drafted tokens each
    (ragged: 1 to that many)."""
    return {"name": name, "op": "tree", "b": b, "lo": lo, "hi": hi, "nodes": nodes, "heads": heads,
            "kv_heads": kv_heads, "d": d, "dtype": dtype, "cache": cache, "page": page, "window": window, "cap": cap,
            "slopes": slopes, "scales": scales, "ragged": ragged}


def _axes(name, b, lo, hi, heads, kv_heads, d, dtype, cache, page, sections, nodes=0, interleaved=False):
    """Prompts of lo..hi tokens, or with `nodes` that many drafted tokens
    behind contexts of lo..hi; sections: rotated pairs of each axis, as text
    (a case's values are plain)."""
    return {"name": name, "op": "axes", "b": b, "lo": lo, "hi": hi, "heads": heads, "kv_heads": kv_heads, "d": d,
            "dtype": dtype, "cache": cache, "page": page, "sections": sections, "nodes": nodes,
            "interleaved": interleaved}


def _fork(name, groups, beams, lo, hi, layers, kv_heads, d, cache, page):
    """groups of `beams` rows over shared contexts of lo..hi tokens; the
    second half of each group loses its place to the first."""
    return {"name": name, "op": "fork", "b": groups, "beams": beams, "lo": lo, "hi": hi, "layers": layers,
            "kv_heads": kv_heads, "d": d, "cache": cache, "page": page}


def _compact(name, b, lo, hi, among, kept, layers, kv_heads, d, cache, page):
    """b contexts of lo..hi tokens; of the `among` tokens behind them (0: of
    their own) `kept` in `among` stay."""
    return {"name": name, "op": "compact", "b": b, "lo": lo, "hi": hi, "among": among, "kept": kept, "layers": layers,
            "kv_heads": kv_heads, "d": d, "cache": cache, "page": page}


def listed():
    return [
        # one short request's prompt, GPT-2-small's heads: latency
        _prompt("prompt_one", 1, 60, 60, 12, 12, 64, "fp16", "fp16", 16),
        # chunks of prompts behind cached tokens, sequences that answer among
        # them with one token each, capped scores and a sliding window
        _prompt("prompt_chunks", 16, 1, 1024, 32, 8, 128, "bf16", "bf16", 16, past=2000, window=1500, cap=50.0),
        # one long prompt
        _prompt("prompt_long", 1, 8192, 8192, 32, 8, 128, "bf16", "bf16", 64),
        # packed documents in 32 bits, a bias by distance, a head of 80
        _prompt("prompt_fp32_documents", 6, 100, 1500, 12, 12, 80, "fp32", "fp32", 16, slopes=True, docs=3),
        # one request's draft, GPT-2-small's heads: latency
        _tree("tree_one", 1, 100, 100, 8, 12, 12, 64, "fp16", "fp16", 16),
        # a serving batch's drafts at every stage of its answers, grouped heads
        _tree("tree_batch", 64, 1, 4096, 16, 32, 8, 128, "bf16", "bf16", 16),
        # wide trees over few long contexts in an 8-bit cache, capped scores
        _tree("tree_long_e4m3", 4, 65536, 65536, 48, 64, 8, 128, "bf16", "e4m3", 64, cap=30.0, scales=True),
        # a batch's drafts are appended: the angle by depth, the place by number
        _axes("axes_draft", 64, 1, 4096, 32, 8, 128, "bf16", "bf16", 16, "64", nodes=16),
        # prompts with video: time, height and width
        _axes("axes_video", 12, 1, 4096, 32, 8, 128, "bf16", "bf16", 64, "16,24,24"),
        # a beam search's step over shared prompts
        _fork("fork_beams", 32, 4, 1, 2048, 4, 8, 128, "bf16", 16),
        # accepted paths of a batch's drafts, all layers
        _compact("compact_draft", 64, 1, 1024, 16, 5, 4, 8, 128, "bf16", 16),
        # half of every long context is evicted
        _compact("compact_evict", 8, 4096, 16384, 0, 0, 2, 8, 128, "bf16", 64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "tree", "tree", "axes", "fork", "compact"])
    heads, kv_heads = rng.choice([(12, 12), (32, 8), (64, 8), (16, 1), (8, 8), (28, 4), (5, 5)])
    d = rng.choice([64, 80, 96, 112, 128, 128, 256])
    dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"),
                               ("fp16", "e4m3"), ("fp32", "fp32")])
    page = rng.choice([16, 16, 32, 64, 128, 48])
    scales = cache == "e4m3" and rng.random() < 0.5
    if op == "prompt":
        b = _log_int(rng, 1, 32)
        # the padded plain form holds every head's scores in 32 bits
        hi = _log_int(rng, 1, min(8192, int((1.5e9 / (b * heads)) ** 0.5)))
        past = rng.choice([0, _log_int(rng, 1, max(1, min(8192, int(1.5e9 / (b * heads * hi)) - hi)))])
        total = past + hi
        case = _prompt("", b, rng.randint(1, hi), hi, heads, kv_heads, d, dtype, cache, page, past=past,
                       window=rng.choice([0, 0, rng.randint(1, total)]), cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                       slopes=rng.random() < 0.3, prefix=rng.choice([0, 0, rng.randint(1, 8)]),
                       docs=rng.choice([0, 0, rng.randint(1, 9)]), scales=scales)
    elif op == "tree":
        b = _log_int(rng, 1, 128)
        nodes = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, min(65536, int(1.5e9 / (b * heads * nodes)), 300_000_000 // (b * kv_heads * d)))
        case = _tree("", b, rng.randint(0, hi), hi, nodes, heads, kv_heads, d, dtype, cache, page,
                     window=rng.choice([0, 0, rng.randint(1, hi)]), cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                     slopes=rng.random() < 0.3, scales=scales, ragged=rng.random() < 0.5)
    elif op == "axes":
        nodes = rng.choice([0, _log_int(rng, 1, 64)])
        b = _log_int(rng, 1, 64 if nodes else 16)
        hi = _log_int(rng, 1, 2048)
        rot = rng.choice([d, d, d // 2])
        count, left, sections = rng.randint(1, 4), rot // 2, []
        for i in range(count):   # any cut of the pairs; some axes may have none
            sections.append(left if i == count - 1 else rng.randint(0, left))
            left -= sections[-1]
        case = _axes("", b, rng.randint(1, hi), hi, heads, kv_heads, d, dtype, cache, page,
                     ",".join(map(str, sections)), nodes=nodes, interleaved=rng.random() < 0.3)
    else:
        layers = rng.randint(1, 4)
        if op == "fork":
            beams = rng.choice([2, 4, 8])
            case = _fork("", _log_int(rng, 1, 64), beams, 1, _log_int(rng, 1, 2048), layers, min(kv_heads, 8), d, cache,
                         page)
        else:
            among = rng.choice([0, _log_int(rng, 1, 64)])
            hi = _log_int(rng, 1, 8192)
            case = _compact("", _log_int(rng, 1, 16), rng.randint(1, hi), hi, among,
                            rng.randint(0, among), layers, min(kv_heads, 8), d, cache, page)
    del case["name"]
    return case


def _lengths(case):
    """The batch's lengths in ascending order: spread evenly over lo..hi."""
    b, lo, hi = case["b"], case["lo"], case["hi"]
    return [hi] if b == 1 else [lo + (hi - lo) * i // (b - 1) for i in range(b)]


def _nodes(case):
    """Drafted tokens of each sequence."""
    b, n = case["b"], case["nodes"]
    return [1 + (n - 1) * i // max(1, b - 1) for i in range(b)] if case.get("ragged") and b > 1 else [n] * b


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _random(gen, dtype, *shape):
    return torch.randn(*shape, device="cuda", generator=gen).to(TYPES[dtype])


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pages(lengths, page, gen):
    """A block table (-1 behind a sequence's last page) that deals pages out in
    random order, and the number of pages, three of them unused."""
    counts = [-(-n // page) for n in lengths]
    total = sum(counts) + 3
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    width = max(counts) + 1
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(width, device="cuda")[None, :] < torch.tensor(counts, device="cuda")[:, None]
    table[used] = order[:sum(counts)]
    return table, total


def _cache(case, n_pages, gen):
    """Keys and values (page, slot, head, d), a head's slots of one page next
    to each other in memory."""
    return {n: _random(gen, case["cache"], n_pages, case["kv_heads"], case["page"], case["d"]).transpose(1, 2)
            for n in ("k", "v")}


def _slopes(heads):
    return 2.0 ** (-8.0 * torch.arange(1, heads + 1, device="cuda", dtype=torch.float32) / heads)


def _drafts(counts, gen):
    """Trees end to end: every node's depth and the bits of its ancestors and
    itself.  A node's parent is one of the four before it, or none."""
    n = max(counts)
    rank = torch.arange(n, device="cuda")
    back = torch.randint(1, 5, (len(counts), n), device="cuda", generator=gen)
    parent = rank - torch.minimum(back, rank + 1)                      # (b, node), -1: none
    # a node's ancestors: its parent's and the parent, a level at a time
    sees = torch.eye(n, dtype=torch.bool, device="cuda").expand(len(counts), n, n)
    step = torch.nn.functional.one_hot(parent.clamp(min=0), n).bool() & (parent >= 0)[..., None]
    step = (step | torch.eye(n, dtype=torch.bool, device="cuda")).float()
    for _ in range(max(1, math.ceil(math.log2(n + 1)))):
        step = (torch.matmul(step, step) > 0).float()
    sees = step > 0
    words = (n + 31) // 32
    bits = torch.zeros(len(counts), n, words * 32, dtype=torch.int64, device="cuda")
    bits[..., :n] = sees
    mask = (bits.view(len(counts), n, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    mask = torch.where(mask >= 2 ** 31, mask - 2 ** 32, mask).to(torch.int32)
    kept = rank[None, :] < torch.tensor(counts, device="cuda")[:, None]
    return (sees.sum(-1) - 1).to(torch.int32)[kept].contiguous(), mask[kept].contiguous()


def _rope(n_pos, rot):
    half = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-2.0 * half / rot)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def _dealt(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lengths = _lengths(case)
    order = torch.randperm(len(lengths), generator=gen, device="cuda").tolist()
    return gen, [lengths[i] for i in order]


def prepare(case, seed):
    gen, lengths = _dealt(case, seed)
    s = {"case": case}
    {"prompt": _prepare_attention, "tree": _prepare_attention, "axes": _prepare_axes, "fork": _prepare_fork,
     "compact": _prepare_compact}[case["op"]](s, case, gen, lengths)
    return s


def _prepare_attention(s, case, gen, lengths):
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "prompt":
        new, total = lengths, [case["past"] + n for n in lengths]
        s["len"] = _ints(total)
        if case["prefix"]:
            s["prefix_len"] = s["len"] // case["prefix"]
        if case["docs"]:
            n, docs = s["len"].long(), case["docs"]
            pos = torch.cat([torch.arange(t - m, t, device="cuda") for m, t in zip(new, total)])
            of = torch.repeat_interleave(n, _ints(new))
            # a document i of n tokens begins at n * i // docs
            edges = of[:, None] * torch.arange(docs, device="cuda") // docs
            s["first_key"] = torch.where(edges <= pos[:, None], edges, 0).amax(1).to(torch.int32)
    else:
        new = _nodes(case)
        total = [n + m for n, m in zip(lengths, new)]
        s["len"] = _ints(lengths)
        s["depth"], s["mask"] = _drafts(new, gen)
    s["start"] = _ints([sum(new[:i]) for i in range(len(new) + 1)])
    s["table"], n_pages = _pages(total, case["page"], gen)
    s["cache"] = _cache(case, n_pages, gen)
    s["q"] = (2 * torch.randn(sum(new), heads, d, device="cuda", generator=gen)).to(TYPES[case["dtype"]])
    s["out"] = torch.empty_like(s["q"])
    s["most"] = max(total), max(new)
    s["slopes"] = _slopes(heads) if case["slopes"] else None
    if case["scales"]:
        s["cache"]["k_scale"], s["cache"]["v_scale"] = (0.5 + torch.rand(kv_heads, device="cuda", generator=gen)
                                                        for _ in range(2))


def _prepare_axes(s, case, gen, lengths):
    sections = [int(x) for x in case["sections"].split(",")]
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["d"]
    if case["nodes"]:
        new = [case["nodes"]] * len(lengths)
        depth, _ = _drafts(new, gen)
    else:
        new = lengths
    n = torch.tensor(new, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), n)
    i = torch.arange(sum(new), device="cuda") - (torch.cumsum(n, 0) - n)[seq]
    past = _ints(lengths)[seq] if case["nodes"] else torch.zeros_like(i)
    s["seq"], s["slot"] = seq.to(torch.int32), (past + i).to(torch.int32)
    if case["nodes"]:
        pos = [past + depth] * len(sections)
    else:
        # frames of 16 x 24 patches: the first axis is the frame, the others a patch's place in it
        pos = [i // 384 + 1, i % 384 // 24, i % 24, i][:len(sections)]
    s["pos"] = torch.stack(pos, dim=1).to(torch.int32)
    s["sections"] = sections
    s["table"], n_pages = _pages([m + (p if case["nodes"] else 0) for m, p in zip(new, lengths)], case["page"], gen)
    s["cache"] = _cache(case, n_pages, gen)
    # the three are parts of one projection's output
    qkv = _random(gen, case["dtype"], seq.numel(), heads + 2 * kv_heads, d)
    s["q"], s["new_k"], s["new_v"] = qkv.split([heads, kv_heads, kv_heads], dim=1)
    s["q_out"] = torch.empty(seq.numel(), heads, d, dtype=qkv.dtype, device="cuda")
    s["rope"] = _rope(max(lengths) + 64, 2 * sum(sections))


def _prepare_fork(s, case, gen, lengths):
    # a group's rows share the pages of the whole context and have their own last page
    b, beams, page = case["b"], case["beams"], case["page"]
    rows = b * beams
    full = [n // page for n in lengths]
    rest = [n % page > 0 for n in lengths]
    total = sum(full) + beams * sum(rest)
    n_pages = total + rows + 5          # some are free
    order = torch.randperm(n_pages, generator=gen, device="cuda")
    width = max(full) + 2
    col = torch.arange(width, device="cuda")
    f, r = torch.tensor(full, device="cuda"), torch.tensor(rest, device="cuda").long()
    first = torch.cumsum(f, 0) - f
    table = torch.where(col < f[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1)], -1)
    table = table[:, None, :].repeat(1, beams, 1)
    own_page = sum(full) + (torch.cumsum(r, 0) - r)[:, None] * beams + torch.arange(beams, device="cuda")
    last = (col == f[:, None]) & (r[:, None] > 0)
    table = torch.where(last[:, None, :], order[own_page.clamp(max=n_pages - 1)][:, :, None], table)
    s["table"] = table.reshape(rows, width).to(torch.int32)
    s["held"] = torch.repeat_interleave(f + r, beams).to(torch.int32)
    s["len"] = torch.repeat_interleave(torch.tensor(lengths, device="cuda"), beams).to(torch.int32)
    used = s["table"][s["table"] >= 0].long()
    s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda").index_add_(
        0, used, torch.ones_like(used, dtype=torch.int32))
    s["free"] = _bits(s["refs"] == 0)
    group = torch.arange(b, device="cuda")[:, None] * beams
    half = torch.arange(beams // 2, device="cuda")
    s["lose"] = (group + beams // 2 + half).flatten().to(torch.int32)
    s["win"] = (group + torch.randint(0, beams // 2, (b, beams // 2), device="cuda", generator=gen)).flatten().to(torch.int32)
    s["none"] = torch.zeros_like(s["lose"])
    s["fork_status"], s["status"] = torch.zeros_like(s["lose"]), torch.zeros_like(s["len"])
    s["next"] = s["len"] + 1
    s["layers"] = [_cache(case, n_pages, gen) for _ in range(case["layers"])]


def _bits(flags):
    """Truth values as bits of 32-bit words."""
    x = torch.zeros((flags.numel() + 31) // 32 * 32, dtype=torch.int64, device="cuda")
    x[:flags.numel()] = flags
    x = (x.view(-1, 32) << torch.arange(32, device="cuda")).sum(1)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


def _prepare_compact(s, case, gen, lengths):
    if case["among"]:
        total, start = [n + case["among"] for n in lengths], lengths
        count, among = [case["kept"]] * len(lengths), [case["among"]] * len(lengths)
    else:
        total, start, count, among = lengths, [0] * len(lengths), [n // 2 for n in lengths], lengths
    width, most = max(1, max(count)), max(among)
    order = torch.rand(len(lengths), most, device="cuda", generator=gen)
    order = order.masked_fill(torch.arange(most, device="cuda") >= _ints(among)[:, None], 2.0).argsort(1)[:, :width]
    order = torch.where(torch.arange(width, device="cuda") < _ints(count)[:, None], order, most)
    s["keep"] = order.sort(1).values.to(torch.int32).contiguous()
    s["count"], s["start"] = _ints(count), _ints(start)
    s["table"], n_pages = _pages(total, case["page"], gen)
    s["layers"] = [_cache(case, n_pages, gen) for _ in range(case["layers"])]


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"prompt": _plain_attention, "tree": _plain_attention, "axes": _plain_axes, "fork": _plain_fork,
            "compact": _plain_compact}[op](s)


def _own(s, op):
    from paper_2111_05426_amd import ops
    case = s["case"]
    if op in ("prompt", "tree"):
        if "workspace" not in s:
            s["workspace"] = ops.alloc_prompt_attention_workspace(s["q"].shape[0], case["b"], case["heads"],
                                                                  case["kv_heads"], case["d"])
        if op == "prompt":
            ops.dsim_prompt_attention(s["q"], s["cache"], s["table"], s["start"], s["len"], s["out"],
                                      window=case["window"], cap=case["cap"], slopes=s["slopes"],
                                      prefix_len=s.get("prefix_len"), first_key=s.get("first_key"),
                                      workspace=s["workspace"])
        else:
            ops.dsim_tree_attention(s["q"], s["cache"], s["table"], s["start"], s["len"], s["mask"], s["out"],
                                    depth=s["depth"], window=case["window"], cap=case["cap"], slopes=s["slopes"],
                                    workspace=s["workspace"])
        return {"out": s["out"]}
    if op == "axes":
        ops.dsim_kv_append_axes(s["cache"], s["table"], s["new_k"], s["new_v"], s["seq"], s["slot"], s["pos"],
                                s["rope"], sections=s["sections"], interleaved=case["interleaved"], q=s["q"],
                                q_out=s["q_out"])
        return {"k": s["cache"]["k"], "v": s["cache"]["v"], "q": s["q_out"]}
    if op == "compact":
        ops.dsim_kv_compact(s["layers"], s["table"], s["start"], s["keep"], s["count"])
        return {"layers": s["layers"]}
    pool = {"refs": s["refs"], "free": s["free"], "held": s["held"]}
    ops.dsim_kv_release(pool, s["table"], case["page"], s["lose"], s["none"])
    ops.dsim_kv_fork(s["layers"], pool, s["table"], s["len"], s["win"], s["lose"], s["fork_status"])
    ops.dsim_kv_reserve(pool, s["table"], case["page"], s["len"], s["next"], s["status"])
    return _fork_outputs(s)


def _fork_outputs(s):
    return {n: s[n] for n in ("table", "refs", "free", "held", "len", "fork_status", "status", "layers")}


def _gathered(x, slot, page):
    """Rows (b, key, head, d) of the cache in 32 bits; slot: places by number."""
    raw = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
    return raw.transpose(1, 2)[slot // page, :, slot % page].view(x.dtype).float()


def _plain_attention(s):
    case = s["case"]
    heads, kv_heads, d, page, b = (case[k] for k in ("heads", "kv_heads", "d", "page", "b"))
    group, (keys_most, new_most) = heads // kv_heads, s["most"]
    tree = case["op"] == "tree"
    j = torch.arange(keys_most, device="cuda")
    i = torch.arange(new_most, device="cuda")
    new = (s["start"][1:] - s["start"][:-1])[:, None]                     # (b, 1)
    there = i < new                                                       # (b, i)
    token = (s["start"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1).long()
    length = s["len"][:, None]
    cached = j[None, :] < length                                          # (b, key): not a drafted one
    if tree:
        node = (j[None, :] - length).clamp(min=0, max=new_most - 1)       # (b, key)
        depth = s["depth"][token]
        at = length + depth                                               # (b, i): positions
        key_at = torch.where(cached, j, length + depth.gather(1, node))
        word = s["mask"][token].gather(2, (node // 32)[:, None, :].expand(-1, new_most, -1))
        drafted = (word >> (node % 32)[:, None, :]) & 1 > 0
        valid = torch.where(cached[:, None, :], torch.ones_like(drafted), drafted & (j < length + new)[:, None, :])
        if case["window"]:
            valid &= (j > at[:, :, None] - case["window"]) | ~cached[:, None, :]
    else:
        at = length - new + i
        key_at = j.expand(b, -1)
        upto = at + 1
        if case["prefix"]:
            upto = torch.maximum(upto, s["prefix_len"][:, None])
        valid = (j < upto[:, :, None]) & cached[:, None, :]
        if case["window"]:
            valid &= j > at[:, :, None] - case["window"]
        if case["docs"]:
            valid &= j >= s["first_key"][token][:, :, None]
    valid = valid & there[:, :, None]
    slot = s["table"].long().clamp(min=0)[:, j // page] * page + j % page
    k, v = _gathered(s["cache"]["k"], slot, page), _gathered(s["cache"]["v"], slot, page)
    q = s["q"].float()[token].view(b, new_most, kv_heads, group, d).permute(0, 2, 3, 1, 4).reshape(
        b, kv_heads, group * new_most, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(d ** -0.5).view(
        b, kv_heads, group, new_most, keys_most)
    if case["scales"]:
        score *= s["cache"]["k_scale"][:, None, None, None]
    if case["cap"]:
        score.div_(case["cap"]).tanh_().mul_(case["cap"])
    if case["slopes"]:
        distance = (at[:, :, None] - key_at[:, None, :]).abs().float()    # (b, i, key)
        score -= s["slopes"].view(kv_heads, group, 1, 1) * distance[:, None, None]
    score.masked_fill_(~valid[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    score.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(b, kv_heads, group * new_most, keys_most), v.transpose(1, 2).contiguous())
    out = out.view(b, kv_heads, group, new_most, d) / torch.where(total == 0.0, 1.0, total)
    if case["scales"]:
        out = out * s["cache"]["v_scale"][:, None, None, None]
    out = out.permute(0, 3, 1, 2, 4).reshape(b, new_most, heads, d)
    s["out"].copy_(out[there])
    return {"out": s["out"]}


def _turned(x, s):
    """x (token, head, d) in 32 bits, its pairs rotated by their axes' positions."""
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device="cuda"),
                                   torch.tensor(s["sections"], device="cuda"))
    half = axis.numel()
    rot = 2 * half
    pos = s["pos"].long()[:, axis]                                         # (token, pair)
    pair = torch.arange(half, device="cuda")
    c, sn = s["rope"][pos, pair][:, None], s["rope"][pos, half + pair][:, None]
    x = x.float()
    if s["case"]["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * sn, b * c + a * sn], dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:rot]
        y = torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_axes(s):
    page = s["case"]["page"]
    slot = s["slot"].long()
    at = s["table"][s["seq"].long(), slot // page].long(), slot % page
    for cache, x in ((s["cache"]["k"], _turned(s["new_k"], s)), (s["cache"]["v"], s["new_v"].float())):
        if cache.dtype == torch.float8_e4m3fn:   # values beyond the type's range become its largest
            cache.view(torch.uint8)[at] = x.clamp(-448.0, 448.0).to(cache.dtype).view(torch.uint8)
        else:
            cache[at] = x.to(cache.dtype)
    s["q_out"].copy_(_turned(s["q"], s))
    return {"k": s["cache"]["k"], "v": s["cache"]["v"], "q": s["q_out"]}


def _count(refs, pages, by):
    refs.index_add_(0, pages, torch.full_like(pages, by, dtype=torch.int32))


def _plain_fork(s):
    page, table, refs = s["case"]["page"], s["table"], s["refs"]
    col = torch.arange(table.shape[1], device="cuda")
    lose, win = s["lose"].long(), s["win"].long()
    # release
    rows = table[lose]
    _count(refs, rows[col < s["held"][lose][:, None]].long(), -1)
    table[lose] = torch.where(col < s["held"][lose][:, None], -1, rows)
    s["held"][lose] = 0
    # fork: whole pages are shared, a page that ends in the middle is copied
    n = s["len"][win]
    whole, rest = n // page, n % page
    shared = col < whole[:, None]
    _count(refs, table[win][shared].long(), 1)
    ends = rest > 0
    fresh = torch.nonzero(refs == 0).flatten()[:int(ends.sum())].to(torch.int32)
    taken = torch.zeros_like(s["lose"]).masked_scatter_(ends, fresh)
    _count(refs, fresh.long(), 1)
    last = (col == whole[:, None]) & ends[:, None]
    before = table[win]
    table[lose] = torch.where(shared, before, torch.where(last, taken[:, None], table[lose]))
    src = before.gather(1, whole[:, None].long().clamp(max=table.shape[1] - 1))[:, 0].long()[ends]
    slots = torch.arange(page, device="cuda") < rest[ends][:, None]
    pair, slot = torch.nonzero(slots, as_tuple=True)
    for layer in s["layers"]:
        for x in (layer["k"], layer["v"]):
            raw = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
            raw[fresh.long()[pair], slot] = raw[src[pair], slot]
    s["held"][lose] = whole + ends.to(torch.int32)
    s["len"][lose] = n
    # reserve
    need = (s["next"] + page - 1) // page - s["held"]
    fresh = torch.nonzero(refs == 0).flatten()[:int(need.sum())].to(torch.int32)
    table[(col >= s["held"][:, None]) & (col < (s["held"] + need)[:, None])] = fresh
    _count(refs, fresh.long(), 1)
    s["held"] += need
    s["free"].copy_(_bits(refs == 0))
    s["fork_status"].zero_()
    s["status"].zero_()
    return _fork_outputs(s)


def _plain_compact(s):
    page, table = s["case"]["page"], s["table"].long()
    i = torch.arange(s["keep"].shape[1], device="cuda")
    used = i < s["count"][:, None]
    seq = torch.nonzero(used, as_tuple=True)[0]
    new, old = (s["start"][:, None] + i)[used], (s["start"][:, None] + s["keep"]).long()[used]
    to, from_ = (table[seq, new // page], new % page), (table[seq, old // page], old % page)
    for layer in s["layers"]:
        for x in (layer["k"], layer["v"]):
            raw = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
            raw[to] = raw[from_]
    return {"layers": s["layers"]}


# ---------------------------------------------------------------------------
# Work and exact results
# ---------------------------------------------------------------------------
def work(case):
    lengths = _lengths(case)
    op = case["op"]
    kv_heads, d = case["kv_heads"], case["d"]
    row = 2 * kv_heads * d * SIZE[case["cache"]]         # a token's key and value
    if op == "fork":
        losers = case["beams"] // 2
        rest = sum(n % case["page"] for n in lengths)
        full = sum(n // case["page"] for n in lengths)
        # of each loser: its row of the table read, cleared and written, its pages counted down and up
        return {"bytes": losers * (2 * row * case["layers"] * rest + 28 * full) + 40 * case["b"] * case["beams"],
                "flops": 0}
    if op == "compact":
        kept = sum(case["kept"] if case["among"] else n // 2 for n in lengths)
        return {"bytes": kept * (2 * row * case["layers"] + 4) + 12 * case["b"], "flops": 0}
    heads = case["heads"]
    if op == "axes":
        tokens = case["nodes"] * case["b"] if case["nodes"] else sum(lengths)
        rot = 2 * sum(int(x) for x in case["sections"].split(","))
        axes = case["sections"].count(",") + 1
        values = tokens * d * (2 * heads * SIZE[case["dtype"]] + 2 * kv_heads * (SIZE[case["dtype"]] + SIZE[case["cache"]]))
        return {"bytes": values + max(lengths) * rot * 4 + tokens * (8 + 4 * axes),
                "flops": 3 * tokens * rot * (heads + kv_heads)}
    if op == "tree":
        new = _nodes(case)
        tokens = sum(new)
        seen = [min(n, case["window"] or n) for n in lengths]
        pairs = sum(m * (n + 1) for m, n in zip(new, seen))
        keys = sum(seen) + tokens
    else:
        tokens = sum(lengths)
        pairs, keys = 0, 0
        for n in lengths:
            lo, hi = _intervals(case, n)
            pairs += int((hi - lo).clamp(min=0).sum())
            keys += int((hi - lo.amin()).clamp(min=0).amax())
    return {"bytes": keys * row + 2 * tokens * heads * d * SIZE[case["dtype"]], "flops": 4 * pairs * heads * d}


def _intervals(case, new):
    """First key and end of the keys of each of a sequence's new tokens."""
    total = case["past"] + new
    p = torch.arange(case["past"], total)
    hi = p + 1
    lo = torch.zeros_like(p)
    if case["prefix"]:
        hi = hi.clamp(min=total // case["prefix"])
    if case["window"]:
        lo = (p + 1 - case["window"]).clamp(min=0)
    if case["docs"]:
        edges = torch.tensor([total * i // case["docs"] for i in range(case["docs"])])
        lo = torch.maximum(lo, edges[torch.searchsorted(edges, p, right=True) - 1])
    return lo, hi


def exact(case, seed):
    op = case["op"]
    if op == "fork":
        return None      # whole numbers, and rows that are copied as they are
    s = prepare(case, seed)
    return {"prompt": _exact_attention, "tree": _exact_attention, "axes": _exact_axes,
            "compact": _exact_compact}[op](case, s)


def _exact_attention(case, s):
    heads, kv_heads, d, page = case["heads"], case["kv_heads"], case["d"], case["page"]
    group = heads // kv_heads
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    start, length = s["start"].tolist(), s["len"].tolist()
    for b in range(case["b"]):
        new = start[b + 1] - start[b]
        rows = slice(start[b], start[b + 1])
        total = length[b] + new if case["op"] == "tree" else length[b]
        j = torch.arange(total, device="cuda")
        if case["op"] == "tree":
            ctx = length[b]
            depth = s["depth"][rows].long()
            p, place = ctx + depth, torch.cat([j[:ctx], ctx + depth])
            bit = torch.arange(new, device="cuda")
            among = torch.bitwise_right_shift(s["mask"][rows].long()[:, bit // 32], bit % 32) % 2 == 1
            past = torch.ones(new, ctx, dtype=torch.bool, device="cuda")
            if case["window"]:
                past = p[:, None] - j[:ctx] < case["window"]
            allowed = torch.cat([past, among], dim=1)
        else:
            lo, hi = (x.cuda() for x in _intervals(case, new))
            p, place = torch.arange(total - new, total, device="cuda"), j
            allowed = (lo[:, None] <= j) & (j < hi[:, None])
        pages = s["table"][b, :-(-total // page)].long()
        for h in range(kv_heads):
            k = s["cache"]["k"][:, :, h][pages].double().flatten(0, 1)[:total]
            v = s["cache"]["v"][:, :, h][pages].double().flatten(0, 1)[:total]
            if case["scales"]:
                k, v = k * s["cache"]["k_scale"][h].double(), v * s["cache"]["v_scale"][h].double()
            for g in range(group):
                score = s["q"][rows, h * group + g].double() @ k.t().contiguous() / math.sqrt(d)
                if case["cap"]:
                    score = case["cap"] * torch.tanh(score / case["cap"])
                if case["slopes"]:
                    score = score - s["slopes"][h * group + g].double() * (p[:, None] - place).abs()
                score[~allowed] = -math.inf
                weight = torch.softmax(score, dim=1)
                weight[~allowed.any(1)] = 0.0
                out[rows, h * group + g] = weight @ v
    return {"out": out}


def _exact_axes(case, s):
    half = sum(s["sections"])
    rot = 2 * half
    rope = s["rope"].double()
    columns, first = [], 0
    for axis, n in enumerate(s["sections"]):
        at = rope[s["pos"][:, axis].long()]
        columns.append(torch.complex(at[:, first:first + n], at[:, half + first:half + first + n]))
        first += n
    turn = torch.cat(columns, dim=1)[:, None, :]
    turned = []
    for x in (s["q"].double(), s["new_k"].double()):
        head = x[..., :rot].contiguous()
        if case["interleaved"]:
            z = torch.view_as_complex(head.view(*head.shape[:-1], half, 2)) * turn
            head = torch.view_as_real(z).reshape(head.shape)
        else:
            z = torch.complex(*head.chunk(2, dim=-1)) * turn
            head = torch.cat([z.real, z.imag], dim=-1)
        turned.append(torch.cat([head, x[..., rot:]], dim=-1))
    k, v = s["cache"]["k"].double(), s["cache"]["v"].double()
    at = (s["table"].long()[s["seq"].long(), torch.div(s["slot"], case["page"], rounding_mode="floor").long()],
          torch.remainder(s["slot"], case["page"]).long())
    most = 448.0 if case["cache"] == "e4m3" else math.inf
    k.index_put_(at, turned[1].clamp(-most, most))
    v.index_put_(at, s["new_v"].double().clamp(-most, most))
    return {"k": k, "v": v, "q": turned[0]}


def _exact_compact(case, s):
    page = case["page"]
    done = []
    for layer in s["layers"]:
        done.append({})
        for name in ("k", "v"):
            x = layer[name].double()
            for b in range(case["b"]):
                n, first = int(s["count"][b]), int(s["start"][b])
                pages = s["table"][b].clamp(min=0).long()
                old = first + s["keep"][b, :n].long()
                rows = x[pages[old // page], old % page]
                new = torch.arange(first, first + n, device="cuda")
                x[pages[new // page], new % page] = rows
            done[-1][name] = x
    return {"layers": done}
