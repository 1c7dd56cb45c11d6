"""Timed cases of pages that sequences share: what a program that serves samples, beams and requests with one beginning has the 8-bit paged cache do.

Five operators: sequences that become others' beginnings (fork), lengths of a step where sequences share pages (grow), pages copied within a pool or into
another one (copy), pages moved together at the pool's beginning (compact), and attention that reads a page once for all sequences that share it (attn).
``own`` chooses between the library's calls and plain tensor operations on the same tensors:

* values, uint8 [layers, pages, KV heads, 2 (K, V), P * 128]: e4m3 bytes, K [token, channel], V [token / 8, channel, token % 8];
* exponents, int32 [layers, pages, KV heads, 2]: a stored v stands for v * 2^exponent;
* table, int32 [sequences, pages a sequence may have]; lens, int32 [sequences]; free, int32 [1 + pages]: a count and a stack of page ids;
* refs, int32 [pages]: how many sequences hold a page (each at the same place of its table);
* starts, int32 [sequences + 1] and slots, int32 [tokens]: where each sequence's new tokens begin, page * P + offset of each (-1: none);
* copies, int32 [n, 2]: (from, to), -1: none.
"""
import math
import random

import torch

HEAD_DIM = 128
LEAST_EXPONENT = -100

own = False


# ------------------------------------------------------------------------------------------------------------------------------ cases
def _case(name, kind, batch, prompts, context, tail, *, nested=False, new=1, layers=1, kv_heads=8, group=4, page=32, dtype="bf16", sink=0, recent=0, spare=1.25,
          other=False, pad=0, shape=1):
    """prompts: sequences that begin on their own, with up to `context` tokens; the others share the beginning of one of them, or, nested, of any sequence before them;
    tail: most tokens of a sequence's own; new: most new tokens of a sequence; spare: pages of the pool over those that are held; other: copies go into another
    pool; pad: rows behind the last sequence; shape: lengths' seed."""
    case = dict(kind=kind, batch=batch, prompts=prompts, context=context, tail=tail, nested=nested, new=new, layers=layers, kv_heads=kv_heads, group=group, page=page,
                dtype=dtype, sink=sink, recent=recent, spare=spare, other=other, pad=pad, shape=shape)
    return dict(case, name=name) if name else case


def listed():
    return [
        # A step of beam search: 8 beams over a prompt of 2000 tokens go on from the best of them.  Latency counts.
        _case("fork-beams-8", "fork", 8, 1, 2000, 200, nested=True),
        # 256 places of a server: new requests take the beginnings of cached ones, finished ones leave.
        _case("fork-server-256", "fork", 256, 16, 8192, 600, page=16),
        # The new tokens of 16 samples that share a prompt: most have to leave the page that they share first.
        _case("grow-samples-16", "grow", 16, 1, 8000, 30),
        # 256 places: chunks of prompts, single tokens, drafts taken back, finished requests whose pages others still hold.
        _case("grow-server-256", "grow", 256, 16, 8192, 600, nested=True, new=512, page=16),
        # The shared last pages of 16 samples, all 32 layers.
        _case("copy-samples-16", "copy", 16, 1, 1000, 1, layers=32),
        # A pool of 131072 tokens that has become too small: its pages into a larger one, 4 layers.
        _case("copy-pool-128k", "copy", 4, 4, 32768, 1, layers=4, page=64, other=True),
        # What 8 requests have left of a small pool, together at its beginning.
        _case("compact-8", "compact", 8, 2, 2000, 200, spare=1.6),
        # The same of 256 places with shared beginnings.
        _case("compact-server-256", "compact", 256, 16, 8192, 600, page=16, spare=1.6),
        # The smallest attention: one layer in fp32, one query head per KV head, 4 samples of a prompt of 1000 tokens -- a model in a debugger, a unit test.
        _case("attn-samples-4-1k-f32", "attn", 4, 1, 1000, 24, group=1, page=16, dtype="f32"),
        # 16 samples of a prompt of 8192 tokens, four layers of a decode step.
        _case("attn-samples-16-8k", "attn", 16, 1, 8192, 512, layers=4),
        # 12 beams whose last 2000 tokens branched again and again, behind a document of 30000, draft tokens, a window.
        _case("attn-beams-12-32k", "attn", 12, 1, 30000, 200, nested=True, new=3, page=16, sink=10, recent=16384, pad=2),
        # 64 requests about one document of 32768 tokens, 8 query heads per KV head.
        _case("attn-document-64-32k", "attn", 64, 1, 32768, 1024, group=8, page=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["fork", "grow", "copy", "compact", "attn", "attn", "attn", "attn"])
        tables = kind in ("fork", "grow", "compact")
        batch = _log_uniform(rng, 1, 256 if tables else 128)
        windows = kind == "attn" and rng.random() < 0.3
        case = _case(None, kind, batch, rng.randint(1, max(1, batch // 4)), _log_uniform(rng, 1, 8192 if kind == "copy" else 65536), _log_uniform(rng, 1, 2048),
                     nested=rng.random() < 0.4, new=_log_uniform(rng, 1, 512 if kind == "grow" else 8) if rng.random() < 0.4 else 1,
                     layers=rng.choice([1, 3, 8, 32] if kind == "copy" else [1, 1, 2, 3]), kv_heads=rng.choice([1, 2, 4, 5, 8, 8, 8]),
                     group=rng.choice([1, 2, 3, 4, 4, 6, 8]), page=rng.choice([16, 32, 64, 128]), dtype="f32" if rng.random() < 0.25 else "bf16",
                     sink=rng.choice([0, 10]) if windows else 0, recent=_log_uniform(rng, 1, 8192) if windows else 0, spare=rng.choice([1.0, 1.25, 1.6]),
                     other=rng.random() < 0.4, pad=rng.choice([0, 0, 3]), shape=rng.randint(1, 1 << 20))
        if _fits(case):
            return case


def _fits(case):
    """No more than the largest listed cases cost, in memory and in time."""
    _, _, lens = _forest(case)
    P, longest = case["page"], max(lens)
    cells = case["layers"] * case["kv_heads"] * HEAD_DIM
    if case["kind"] in ("fork", "grow", "compact"):
        return case["batch"] * _pages(longest, P) <= 1 << 18
    held = len({p for row in _rows(case)[0] for p in row})
    if case["kind"] == "copy":
        return cells * P * held * 2 <= 1 << 30
    heads = case["kv_heads"] * case["group"]
    return (case["batch"] * longest * case["kv_heads"] * HEAD_DIM <= 5 << 29 and heads * case["batch"] * case["new"] * longest <= 1 << 28
            and heads * sum(lens) * case["new"] * case["layers"] <= 9 << 24 and cells * P * held <= 1 << 28)


def _forest(case):
    """Of every sequence: the one whose beginning it shares (-1: none), how many tokens of it, and its length."""
    rng = random.Random(case["shape"])
    parents, keeps, lens = [], [], []
    for b in range(case["batch"]):
        tail = rng.randint(1, case["tail"])
        if b < case["prompts"]:
            parents.append(-1), keeps.append(0)
            lens.append((rng.randint((case["context"] + 1) // 2, case["context"]) if b else case["context"]) + tail)
        elif case["batch"] > 4 and b % 16 == 4:  # a place that no request has now
            parents.append(-1), keeps.append(0), lens.append(0)
        else:
            root = b % case["prompts"]
            parent = rng.randrange(b) if case["nested"] else root
            if lens[parent] == 0:
                parent = root
            least = min(lens[root], lens[parent]) * 9 // 10
            keep = rng.randint(least, lens[parent]) if case["nested"] else min(case["context"], lens[root])
            parents.append(parent), keeps.append(keep), lens.append(keep + tail)
    return parents, keeps, lens


def _rows(case):
    """Pages of every sequence, numbered as they come, and the lengths: shared up to the last full page of the common beginning."""
    parents, keeps, lens = _forest(case)
    P, rows, n = case["page"], [], 0
    for parent, keep, length in zip(parents, keeps, lens):
        row = rows[parent][:keep // P] if parent >= 0 else []
        fresh = _pages(length, P) - len(row)
        rows.append(row + list(range(n, n + fresh)))
        n += fresh
    return rows, lens


def _news(case, lens):
    rng = random.Random(case["shape"] + 1)
    return [min(n, rng.randint(1, case["new"])) for n in lens]


def _pages(n, P):
    return (n + P - 1) // P


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ----------------------------------------------------------------------------------------------------------------------------- inputs
def _normal(shape, scale, dtype, gen):
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * scale if scale is not None else x).to(dtype)


def _pool(case, n_pages, gen):
    """Pages full of tokens, as writing them leaves the pool; K: log-uniform scales of the channels."""
    nl, H, P = case["layers"], case["kv_heads"], case["page"]
    scale = 10.0 ** (2.0 * torch.rand((nl, H, HEAD_DIM), generator=gen, device="cuda") - 1.0)
    values = torch.empty((nl, n_pages, H, 2, P * HEAD_DIM), dtype=torch.uint8, device="cuda")
    exponents = torch.empty((nl, n_pages, H, 2), dtype=torch.int32, device="cuda")
    for layer in range(nl):
        for which in (0, 1):
            x = _normal((n_pages, H, P, HEAD_DIM), scale[layer][:, None, :] if which == 0 else None, torch.float32, gen)
            m, k = torch.frexp(x.abs().amax((2, 3)))
            e = (k - 9 + (m > 0.875)).clamp_min(LEAST_EXPONENT).to(torch.int32)
            x = (x * _power32(-e)[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            if which:
                x = x.view(n_pages, H, P // 8, 8, HEAD_DIM).transpose(3, 4)
            values[layer, :, :, which] = x.reshape(n_pages, H, P * HEAD_DIM)
            exponents[layer, :, :, which] = e
    return values, exponents


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _tables(case, seed):
    """The pool's tables as one array of whole numbers and views of it: table, lens, free, refs.  Pages lie in the pool in any order."""
    rng = random.Random(seed)
    rows, lens = _rows(case)
    B, held = case["batch"], len({p for row in rows for p in row})
    width, n_pages = max(1, max(map(len, rows))) + 2 + _pages(case["new"], case["page"]), max(1, int(math.ceil(held * case["spare"])))
    order = list(range(n_pages))
    rng.shuffle(order)
    table = [[order[p] for p in row] + [-1] * (width - len(row)) for row in rows]
    refs = [0] * n_pages
    for row in rows:
        for p in row:
            refs[order[p]] += 1
    free = [n_pages - held] + order[held:] + [-1] * held
    flat = _ints([p for row in table for p in row] + lens + free + refs)
    return flat, _views(flat, B, width, n_pages), lens


def _views(flat, B, width, n_pages):
    parts = flat.split([B * width, B, 1 + n_pages, n_pages])
    return dict(table=parts[0].view(B, width), lens=parts[1], free=parts[2], refs=parts[3])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    flat, t, lens = _tables(case, seed)
    B, P, (nl, H) = case["batch"], case["page"], (case["layers"], case["kv_heads"])
    n_pages = t["refs"].numel()
    state = dict(case=case, **t)
    live = [b for b in range(B) if lens[b]]
    if case["kind"] == "fork":
        # most places go on from a sequence that does well, some from a part of it, some stay, some are given up
        best = rng.sample(live, max(1, len(live) // 2))
        parent = [b if lens[b] and rng.random() < 0.3 else rng.choice(best) for b in range(B)]
        keep = [-1 if x < 0.7 else 0 if x < 0.85 else rng.randint(1, max(1, lens[p])) for p, x in zip(parent, (rng.random() for _ in parent))]
        state.update(parent=_ints(parent), keep=_ints(keep))
    if case["kind"] == "grow":
        # samples: every other live place takes over, whole, the one before it, whose last page they then share
        shared = [b - 1 if b % 2 and lens[b - 1] else b for b in range(B)]
        if case["prompts"] == 1:
            shared = [0] * B
        _plain_fork(_ints(shared), None, t["table"], t["lens"], t["free"], t["refs"], P)
        have, rng = t["lens"].tolist(), random.Random(case["shape"] + 2)  # as many slots with every seed
        want = [n + rng.randint(1, case["new"]) for n in have]
        if case["new"] > 1:  # a server: some are done, some take drafts back, some wait, some bring one token
            turn = [rng.random() for _ in have]
            want = [0 if x < 0.1 else max(0, n - rng.randint(1, 64)) if x < 0.2 else -1 if x < 0.3 else n + 1 if x < 0.8 else w for w, n, x in zip(want, have, turn)]
        want = [min(w, t["table"].shape[1] * P) for w in want]
        new = sum(max(0, w - n) for w, n in zip(want, have))
        state.update(want=_ints(want), starts=_ints([0] * (B + 1)), slots=_ints([0] * (new + case["pad"])), copies=_ints([[0, 0]] * B))
    if case["kind"] in ("fork", "grow", "compact"):
        state.update(flat=flat, before=flat.clone())
        if case["kind"] == "compact":
            state["moves"] = _ints([[0, 0]] * n_pages)
        return state
    if case["kind"] == "copy":
        n = n_pages if case["other"] else max(1, n_pages // 2)
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        count = n if case["other"] else max(1, min(B, n))
        state["values"], state["exponents"] = _pool(case, n_pages if case["other"] else max(2, n_pages), gen)
        if case["other"]:
            more = n_pages * 3 // 2
            state["to_values"] = torch.zeros((nl, more, H, 2, P * HEAD_DIM), dtype=torch.uint8, device="cuda")
            state["to_exponents"] = torch.zeros((nl, more, H, 2), dtype=torch.int32, device="cuda")
            state["copies"] = torch.stack([order, torch.arange(n_pages, dtype=torch.int32, device="cuda")], 1).contiguous()
        else:  # few sources, as shared pages are, and targets of their own; some places have nothing to copy
            page = torch.randperm(state["values"].shape[1], generator=gen, device="cuda").to(torch.int32)
            to = page[:count]
            source = page[count:] if page.numel() > count else page[:0]
            count = count if source.numel() else 0
            copies = torch.full((B, 2), -1, dtype=torch.int32, device="cuda")
            if count:
                copies[:count, 0] = source[torch.arange(count, device="cuda") % min(4, source.numel())]
                copies[:count, 1] = to
            state["copies"] = copies
        return state
    state["values"], state["exponents"] = _pool(case, n_pages, gen)
    news = _news(case, lens)
    starts = [0]
    for k in news:
        starts.append(starts[-1] + k)
    n_tokens, heads = starts[-1] + case["pad"], H * case["group"]
    state.update(q=_normal((nl, n_tokens, heads, HEAD_DIM), None, _dtype(case), gen), starts=_ints(starts), longest=max(lens), most=max(news),
                 out=torch.zeros((nl, n_tokens, heads, HEAD_DIM), dtype=_dtype(case), device="cuda"))
    return state


# ------------------------------------------------------------------------------------------------------------------------- one pass
_TABLES = ("table", "lens", "free", "refs")


def run(state):
    if own:
        return _own(state)
    s, case = state, state["case"]
    P = case["page"]
    if case["kind"] in ("fork", "grow", "compact"):
        s["flat"].copy_(s["before"])  # the state before the step
    if case["kind"] == "fork":
        _plain_fork(s["parent"], s["keep"], s["table"], s["lens"], s["free"], s["refs"], P)
        return {k: s[k] for k in _TABLES}
    if case["kind"] == "grow":
        _plain_grow(s["want"], s["table"], s["lens"], s["free"], s["refs"], s["starts"], s["slots"], s["copies"], P)
        return {k: s[k] for k in (*_TABLES, "starts", "slots", "copies")}
    if case["kind"] == "compact":
        _plain_compact(s["table"], s["lens"], s["free"], s["refs"], s["moves"], P)
        return {k: s[k] for k in (*_TABLES, "moves")}
    if case["kind"] == "copy":
        to_values, to_exponents = s.get("to_values", s["values"]), s.get("to_exponents", s["exponents"])
        there = s["copies"][:, 0] >= 0
        source, target = s["copies"][there, 0].long(), s["copies"][there, 1].long()
        to_values[:, target] = s["values"][:, source]
        to_exponents[:, target] = s["exponents"][:, source]
        return {"values": to_values.view(torch.float8_e4m3fn), "exponents": to_exponents}
    for layer in range(case["layers"]):
        _plain_attn(s["values"][layer], s["exponents"][layer], s["q"][layer], s["starts"], s["table"], s["lens"], s["out"][layer], s["longest"], s["most"], case)
    return s["out"]


def _own(s):
    from paper_2507_20030_amd import binding
    case = s["case"]
    P = case["page"]
    if case["kind"] in ("fork", "grow", "compact"):
        s["flat"].copy_(s["before"])
    if case["kind"] == "fork":
        binding.iwdft_pages_fork(s["parent"], s["keep"], s["table"], s["lens"], s["free"], s["refs"], P)
        return {k: s[k] for k in _TABLES}
    if case["kind"] == "grow":
        binding.iwdft_pages_resize_shared(s["want"], s["table"], s["lens"], s["free"], s["refs"], s["starts"], s["slots"], s["copies"], P)
        return {k: s[k] for k in (*_TABLES, "starts", "slots", "copies")}
    if case["kind"] == "compact":
        binding.iwdft_pages_compact(s["table"], s["lens"], s["free"], s["refs"], s["moves"], P)
        return {k: s[k] for k in (*_TABLES, "moves")}
    if case["kind"] == "copy":
        to_values, to_exponents = s.get("to_values", s["values"]), s.get("to_exponents", s["exponents"])
        binding.iwdft_pages_copy(s["copies"], s["values"], s["exponents"], to_values, to_exponents)
        return {"values": to_values.view(torch.float8_e4m3fn), "exponents": to_exponents}
    # once a step who shares what, then every layer's attention
    plan = binding.iwdft_pages_plan(s["starts"], s["table"], s["lens"], s["q"].shape[1], s["values"].shape[1], case["kv_heads"], case["kv_heads"] * case["group"], P,
                                    _dtype(case), n_sink=case["sink"], n_recent=case["recent"])
    for layer in range(case["layers"]):
        binding.iwdft_pages_attn_shared(s["values"], s["exponents"], s["q"][layer:layer + 1], plan, s["table"], s["out"][layer:layer + 1], layer=layer)
    return s["out"]


# ------------------------------------------------------------------------------------------------------------------------ plain forms
def _power32(e):
    """2^e from its bits, -126 <= e <= 127."""
    return (e + 127 << 23).view(torch.float32)


def _count(pages, there, n_pages):
    """How often each page is among those."""
    at = torch.where(there, pages, n_pages).flatten().long()
    return torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda").scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:n_pages]


def _give_back(pages, leaves, left, free):
    """Those of the pages that leave which nobody holds any more (left: holders) onto the stack: as if their holders gave them back one by one, from the last page
    of the last sequence on, and each page went with its last holder.  Returns how many."""
    n_pages, index = left.numel(), torch.arange(pages.numel(), device="cuda")
    page = torch.where(leaves, pages, n_pages).flatten().long()
    first = torch.full((n_pages + 1,), pages.numel(), device="cuda").scatter_reduce(0, page, index, "amin")
    goes = (page < n_pages) & (left[page.clamp_max(n_pages - 1)] <= 0) & (first[page] == index)
    released = goes.sum()
    rank = released - goes.cumsum(0)
    stack = torch.cat([free[1:], free[:1]])  # one place more, for what stays
    stack[torch.where(goes, free[0] + rank, n_pages)] = page.to(torch.int32)
    free[1:] = stack[:-1]
    return released


def _plain_fork(parent, keep, table, lens, free, refs, P):
    B, W = table.shape
    n_pages, column = refs.numel(), torch.arange(W, device="cuda")[None, :]
    parent = torch.where((parent < 0) | (parent >= B), torch.arange(B, device="cuda"), parent.long())
    length = lens[parent] if keep is None else torch.where(keep < 0, lens[parent], torch.minimum(keep, lens[parent]))
    was, now = column < _pages(lens, P)[:, None], column < _pages(length, P)[:, None]
    old, new = table.clone(), torch.where(now, table[parent], table)
    refs += _count(new, now, n_pages) - _count(old, was, n_pages)
    free[0] += _give_back(old, was & (~now | (old != new)), refs, free).to(torch.int32)
    table.copy_(new)
    lens.copy_(length)


def _plain_grow(want, table, lens, free, refs, starts, slots, copies, P):
    B, W = table.shape
    n_pages, column = refs.numel(), torch.arange(W, device="cuda")[None, :]
    have = lens.long()
    want = torch.where((want < 0) | (want > W * P), have, want.long())
    down, up = want < have, want > have
    had, get = _pages(have, P), _pages(want, P)
    leaves = (column >= get[:, None]) & (column < had[:, None])
    refs -= _count(table, leaves, n_pages)
    free[0] += _give_back(table, leaves, refs, free).to(torch.int32)
    # a page that others hold too is left before it takes tokens, unless all of them leave it: then the last one stays
    last = table.gather(1, (had - 1).clamp_min(0)[:, None])[:, 0].long()
    shared = up & (have % P != 0) & (refs[last] > 1)
    order, same = torch.arange(B, device="cuda"), (last[:, None] == last[None, :]) & shared[None, :] & shared[:, None]
    stays = shared & (same.sum(1) == refs[last]) & ~(same & (order[None, :] > order[:, None])).any(1)
    leave = shared & ~stays
    need, new = torch.where(up, get - had + leave, 0), torch.where(up, want - have, 0)
    up = up & (new.cumsum(0) <= slots.numel()) & (((need == 0) & ~shared) | (need.cumsum(0) <= free[0]))
    leave, need, new = leave & up, torch.where(up, need, 0), torch.where(up, new, 0)
    # from the top of the stack, in order: the page in place of the shared one, then the others
    first = torch.where(leave, had - 1, had)
    enters = (column >= first[:, None]) & (column < (first + need)[:, None])
    at = free[0] - enters.flatten().cumsum(0)
    page = torch.where(enters, free[1 + at.clamp(0, n_pages - 1)].view(B, W), table)
    free[0] -= need.sum().to(torch.int32)
    refs -= _count(last, leave, n_pages)
    refs += _count(page, enters, n_pages)
    table.copy_(page)
    lens.copy_(torch.where(up | down, want, have))
    copies[:, 0] = torch.where(leave, last, -1)
    copies[:, 1] = torch.where(leave, page.gather(1, (had - 1).clamp_min(0)[:, None])[:, 0], -1)
    starts[0] = 0
    starts[1:] = new.cumsum(0)
    token = torch.arange(slots.numel(), device="cuda")
    owner = torch.searchsorted(starts[1:].long(), token, right=True).clamp_max(B - 1)
    position = have[owner] + token - starts[owner]
    slot = table[owner, (position // P).clamp(0, W - 1)] * P + position % P
    slots.copy_(torch.where(token < starts[-1], slot, -1))


def _plain_compact(table, lens, free, refs, moves, P):
    """The highest held page to the lowest free place, the next ones, while that brings them down."""
    n_pages, index = refs.numel(), torch.arange(refs.numel(), device="cuda")
    held = refs > 0
    n = held.sum()
    down = torch.sort(torch.where(held, n_pages - 1 - index, n_pages))[0]  # held pages from the highest on
    up = torch.sort(torch.where(held, n_pages, index))[0]  # free places from the lowest on
    source = n_pages - 1 - down
    moved = (index < torch.minimum(n, n_pages - n)) & (up < source) & (index < moves.shape[0])
    to = index.clone()
    to[torch.where(moved, source, n_pages - 1)] = torch.where(moved, up, to[n_pages - 1])
    to[n_pages - 1] = torch.where(moved[0] & (source[0] == n_pages - 1), up[0], n_pages - 1)  # where all that does not move has gone
    count = torch.zeros_like(refs).scatter_add_(0, to, refs.clamp_min(0))
    mine = torch.arange(table.shape[1], device="cuda")[None, :] < _pages(lens, P)[:, None]
    table.copy_(torch.where(mine, to[table.clamp(0, n_pages - 1).long()].to(torch.int32), table))
    refs.copy_(count)
    empty = torch.sort(torch.where(count > 0, -1, index), descending=True)[0]  # the lowest on top
    free[1:] = torch.where(index < n_pages - n, empty, free[1:].long()).to(torch.int32)
    free[0] = (n_pages - n).to(torch.int32)
    m = moves.shape[0]
    moves[:, 0] = torch.where(moved, source, -1)[:m]
    moves[:, 1] = torch.where(moved, up, -1)[:m]


def _scaled(x, e):
    half = torch.div(e, 2, rounding_mode="floor")
    return x * _power32(half) * _power32(e - half)


def _tokens(values, exponents, table, n, P):
    """K, V of the first n tokens of every row of the table, of one layer: fp32 [sequences, KV heads, n, 128]."""
    n_pages, H = exponents.shape[:2]
    token, got = torch.arange(n, device="cuda"), []
    page = table[:, token // P].long().clamp(0, n_pages - 1)
    for which in (0, 1):
        store = values[:, :, which]
        store = store.view(n_pages, H, P, HEAD_DIM) if which == 0 else store.view(n_pages, H, P // 8, HEAD_DIM, 8).transpose(3, 4).reshape(n_pages, H, P, HEAD_DIM)
        x = store[page, :, token % P].view(torch.float8_e4m3fn).permute(0, 2, 1, 3).float()
        got.append(_scaled(x, exponents[..., which][page].transpose(1, 2)[..., None]))
    return got


def _plain_attn(values, exponents, q, starts, table, lens, out, longest, most, case):
    n_tokens, heads = q.shape[:2]
    B, H, P = table.shape[0], exponents.shape[1], case["page"]
    G = heads // H
    K, V = _tokens(values, exponents, table, longest, P)
    new = starts[1:] - starts[:-1]
    row, column = torch.arange(most, device="cuda"), torch.arange(longest, device="cuda")
    V.masked_fill_((column[None, :] >= lens[:, None])[:, None, :, None], 0.0)
    pick = (starts[:-1, None] + row[None, :]).clamp_max(n_tokens - 1).long()  # [sequence, its new tokens]
    x = q.float()[pick].view(B, most, H, G, HEAD_DIM).permute(0, 2, 3, 1, 4).reshape(B, H, G * most, HEAD_DIM)
    scores = torch.matmul(x, K.transpose(2, 3).contiguous()).view(B, H, G, most, longest)
    scores *= HEAD_DIM ** -0.5
    position = (lens[:, None] - new[:, None] + row[None, :])[:, :, None]
    visible = column <= position
    if case["recent"]:
        visible &= (column < case["sink"]) | (column > position - case["recent"])
    scores.masked_fill_(~visible[:, None, None], -math.inf)
    scores -= scores.amax(4, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    scores.exp_()
    total = scores.sum(4, keepdim=True)
    y = torch.matmul(scores.view(B, H, G * most, longest), V).view(B, H, G, most, HEAD_DIM)
    y = torch.where(total > 0, y / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, most, heads, HEAD_DIM)
    token = torch.arange(n_tokens, device="cuda")
    owner = torch.searchsorted(starts[1:].contiguous(), token, right=True).clamp_max(B - 1)
    mine = y[owner, (token - starts[owner]).clamp(0, most - 1)].to(out.dtype)
    out.copy_(torch.where((token < starts[-1])[:, None, None], mine, out))


# -------------------------------------------------------------------------------------------------------------------- work, definition
def work(case):
    rows, lens = _rows(case)
    P, H, G, nl, B = case["page"], case["kv_heads"], case["group"], case["layers"], case["batch"]
    entries, held = sum(map(len, rows)), len({p for row in rows for p in row})
    if case["kind"] == "fork":  # entries of the rows that change read and written, about half of them; their pages' counts
        return dict(bytes=4 * (2 * entries + 4 * B), flops=0)
    if case["kind"] == "grow":
        pages = B * (1 + _pages(case["new"], P) // 2)
        return dict(bytes=4 * (4 * pages + 6 * B + B * case["new"] // 2), flops=0)
    if case["kind"] == "compact":  # every entry and every page's count read, what moves written, the free pages written
        n_pages = max(1, int(math.ceil(held * case["spare"])))
        return dict(bytes=4 * (entries + n_pages + (n_pages - held) + 2 * entries // 3), flops=0)
    page_bytes = nl * H * 2 * (P * HEAD_DIM + 4)
    if case["kind"] == "copy":
        n_pages = max(1, int(math.ceil(held * case["spare"])))
        count = n_pages if case["other"] else max(1, min(B, max(1, n_pages // 2)))
        return dict(bytes=page_bytes * (2 * count if case["other"] else count + min(count, 4)), flops=0)
    news, item = _news(case, lens), _dtype(case).itemsize
    pairs, seen = 0, {}
    for row, n, k in zip(rows, lens, news):
        for p in range(n - k, n):
            ranges = [(max(0, p + 1 - case["recent"]), p + 1), (0, min(case["sink"], p + 1))] if case["recent"] else [(0, p + 1)]
            if len(ranges) == 2:
                ranges[1] = (0, min(ranges[1][1], ranges[0][0]))
            for lo, hi in ranges:
                pairs += max(0, hi - lo)
                for j in range(lo // P, _pages(hi, P)) if hi > lo else ():
                    a, b = max(lo - j * P, 0), min(hi - j * P, P)
                    seen[row[j]] = seen.get(row[j], 0) | ((1 << b) - (1 << a))
    tokens = sum(bin(bits).count("1") for bits in seen.values())  # each shared one once
    return dict(bytes=nl * (H * 2 * HEAD_DIM * tokens + 2 * sum(news) * H * G * HEAD_DIM * item), flops=4 * HEAD_DIM * nl * H * G * pairs)


def _grid_values():
    """What the 256 bytes of e4m3 stand for."""
    got = []
    for byte in range(256):
        e, m = byte >> 3 & 15, byte & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v = math.nan if byte & 127 == 127 else v
        got.append(-v if byte & 128 else v)
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def exact(case, seed):
    if case["kind"] not in ("copy", "attn"):
        return None  # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "copy":
        source, target, grid = s["values"], s.get("to_values", s["values"]), _grid_values()
        got = torch.stack([grid[x.int()] for x in target])  # layer by layer
        for a, b in s["copies"].tolist():
            if a >= 0:
                got[:, b] = grid[source[:, a].int()]
        return {"values": got, "exponents": None}
    P, H, G = case["page"], case["kv_heads"], case["group"]
    lens, table, starts = s["lens"].tolist(), s["table"].tolist(), s["starts"].tolist()
    grid, got = _grid_values(), torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for layer in range(case["layers"]):
        for b, n in enumerate(lens):
            if not n:
                continue
            ids = torch.tensor(table[b][:_pages(n, P)], device="cuda")
            power = torch.pow(2.0, s["exponents"][layer, ids].double())  # [page, head, 2]
            raw = grid[s["values"][layer, ids].int()]
            k = (raw[:, :, 0].view(-1, H, P, HEAD_DIM) * power[:, :, 0, None, None]).permute(1, 0, 2, 3).reshape(H, -1, HEAD_DIM)[:, :n]
            v = (raw[:, :, 1].view(-1, H, P // 8, HEAD_DIM, 8).permute(0, 1, 2, 4, 3).reshape(-1, H, P, HEAD_DIM) * power[:, :, 1, None, None])
            v = v.permute(1, 0, 2, 3).reshape(H, -1, HEAD_DIM)[:, :n]
            news = starts[b + 1] - starts[b]
            p, j = torch.arange(n - news, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None, :]
            hidden = j > p
            if case["recent"]:
                hidden = hidden | ((j >= case["sink"]) & (j <= p - case["recent"]))
            rows = slice(starts[b], starts[b + 1])
            for h in range(H):
                x = s["q"][layer, rows, h * G:(h + 1) * G].double()  # [token, head, 128]
                w = (x.reshape(-1, HEAD_DIM) @ k[h].T / math.sqrt(HEAD_DIM)).view(news, G, n)
                w = torch.softmax(w.masked_fill(hidden[:, None, :], -math.inf), dim=2)
                got[layer, rows, h * G:(h + 1) * G] = (w.reshape(-1, n) @ v[h]).view(news, G, HEAD_DIM)
    return got
