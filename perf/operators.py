"""Timed cases of the 8-bit paged cache: what a program that serves requests beside the frequency-domain cache has the library do.

Four operators: the block tables, slot maps and free list of a step from the lengths that its sequences are to have (resize), new tokens
into the pages (write), attention of the new tokens over the pages (attn), and the pages' tokens as the prefill takes them (read).  ``own``
chooses between the library's calls and plain tensor operations on the same tensors:

* values, uint8 [layers, pages, KV heads, 2 (K, V), P * 128]: e4m3 bytes, K [token, channel], V [token / 8, channel, token % 8];
* exponents, int32 [layers, pages, KV heads, 2]: a stored v stands for v * 2^exponent; the smallest one at which the largest finite value
  that entered the page since its first token is no more than 448, at least -100;
* table, int32 [sequences, pages a sequence may have]; lens, int32 [sequences]; free, int32 [1 + pages]: a count and a stack of page ids;
* starts, int32 [sequences + 1] and slots, int32 [tokens]: where each sequence's new tokens begin, page * P + offset of each (-1: none).
"""
import math
import random

import torch

HEAD_DIM = 128
LEAST_EXPONENT = -100

own = False


# ------------------------------------------------------------------------------------------------------------------------------ cases
def _case(name, kind, batch, context, new, *, chunks=0, ragged=True, layers=1, kv_heads=8, group=4, page=32, dtype="bf16", sink=0, recent=0, spare=1.25,
          pad=0, shape=1):
    """new: most new tokens of a sequence; chunks: sequences that bring so many (0: all; the others bring one); ragged: contexts from a quarter of
    `context` on and an idle sequence; spare: pages of the pool over those that the sequences take; pad: rows behind the last sequence; shape: lengths' seed."""
    case = dict(kind=kind, batch=batch, context=context, new=new, chunks=chunks, ragged=ragged, layers=layers, kv_heads=kv_heads, group=group, page=page,
                dtype=dtype, sink=sink, recent=recent, spare=spare, pad=pad, shape=shape)
    return dict(case, name=name) if name else case


def listed():
    return [
        # A decode step of 16 requests in all: a token each, now and then a page.  One launch; latency counts.
        _case("resize-decode-16", "resize", 16, 16384, 1),
        # 256 requests, each with a prompt of up to 2048 more tokens admitted at once.
        _case("resize-prompts-256", "resize", 256, 8192, 2048, page=16),
        # The tokens of that decode step into one layer's pages.
        _case("write-decode-16", "write", 16, 16384, 1, group=8),
        # 8 prompts of up to 8192 tokens into one layer's pages, behind what is there.
        _case("write-prompts-8", "write", 8, 10000, 8192, page=64),
        # The smallest attention: one layer in fp32, one query head per KV head -- a model in a debugger, a unit test, a draft model.
        _case("attn-one-layer-1k-f32", "attn", 1, 1024, 1, ragged=False, group=1, page=16, dtype="f32"),
        # One user of an 8-billion-parameter model at 8192 tokens, one layer of a decode step.
        _case("attn-8k", "attn", 1, 8192, 1, ragged=False),
        # A served batch, 8 query heads per KV head, contexts of 4096 to 16384 tokens.
        _case("attn-batch16-16k", "attn", 16, 16384, 1, group=8, pad=3),
        # One user with a document of 131072 tokens whose draft model proposes five tokens.
        _case("attn-draft-128k", "attn", 1, 131072, 5, ragged=False, page=128),
        # A prompt of 8000 tokens at once: every token sees those before it.
        _case("attn-prompt-8k", "attn", 1, 8000, 8000, ragged=False, page=64),
        # A served step: two requests bring the next 1000 tokens of their prompts, six decode.  The paper's sinks, a window of 4096.
        _case("attn-mixed-window-16k", "attn", 8, 16384, 1000, chunks=2, sink=10, recent=4096),
        # A context of 8192 tokens and the paper's windows to be compressed: all 32 layers as the prefill takes them.
        _case("read-8k", "read", 1, 8192 + 60, 0, ragged=False, layers=32),
        # Eight short requests in fp32, one layer, to look at.
        _case("read-ragged-1k-f32", "read", 8, 1000, 0, page=16, dtype="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["resize", "write", "attn", "attn", "attn", "read"])
        batch, page = _log_uniform(rng, 1, 256 if kind == "resize" else 64), rng.choice([16, 32, 64, 128])
        context = _log_uniform(rng, 1, 131072)
        new, chunks = 1, 0
        if kind != "read" and rng.random() < 0.6:
            new = _log_uniform(rng, 1, 16 if rng.random() < 0.4 else min(context, 8192))
            chunks = rng.randint(0, min(batch, 3))
        windows = kind == "attn" and rng.random() < 0.3
        case = _case(None, kind, batch, context, new, chunks=chunks, ragged=batch > 1 and rng.random() < 0.8, layers=rng.choice([1, 1, 1, 2, 5]),
                     kv_heads=rng.choice([1, 2, 4, 5, 8, 8, 8]), group=rng.choice([1, 2, 3, 4, 4, 6, 8]), page=page,
                     dtype="f32" if rng.random() < 0.25 else "bf16", sink=rng.choice([0, 10]) if windows else 0,
                     recent=_log_uniform(rng, 1, 8192) if windows else 0, spare=0.9 if kind == "resize" and rng.random() < 0.25 else 1.25,
                     pad=rng.choice([0, 0, 3]), shape=rng.randint(1, 1 << 20))
        if _fits(case):
            return case


def _fits(case):
    """No more than the largest listed cases cost, in memory and in time."""
    lens, news = _lengths(case)
    longest, most = max(lens), max(news)
    cells = case["layers"] * case["kv_heads"] * HEAD_DIM * case["batch"]
    tokens, new_tokens = sum(lens), sum(news)
    if case["kind"] == "resize":
        return case["batch"] * longest <= 1 << 22 and new_tokens >= 1
    if case["kind"] == "write":
        return cells // case["batch"] * tokens <= 1 << 27 and new_tokens >= 1
    if case["kind"] == "read":
        return tokens >= 1 and cells * longest <= 1 << 28
    heads = case["layers"] * case["kv_heads"] * case["group"]
    pairs = sum(_visible_counts(n, k, case["sink"], case["recent"])[0] for n, k in zip(lens, news))
    return new_tokens >= 1 and cells * longest <= 1 << 28 and heads * case["batch"] * most * longest <= 1 << 32 and heads * pairs <= 1 << 30


def _lengths(case):
    """Length of every sequence after the step, and its new tokens among them."""
    rng = random.Random(case["shape"])
    lens, news = [], []
    for b in range(case["batch"]):
        n = rng.randint(max(1, case["context"] // 4), case["context"]) if case["ragged"] else case["context"]
        long = case["chunks"] == 0 or b < case["chunks"]
        k = min(n, (rng.randint((case["new"] + 1) // 2, case["new"]) if case["ragged"] else case["new"]) if long else 1)
        if case["ragged"] and case["batch"] > 4 and b == 3:  # a place that no request has now
            n = k = 0
        lens.append(n)
        news.append(k)
    return lens, news


def _pages(n, P):
    return (n + P - 1) // P


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ----------------------------------------------------------------------------------------------------------------------------- inputs
def _normal(shape, scale, dtype, gen):
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * scale if scale is not None else x).to(dtype)


def _pool(case, n_pages, scale, gen):
    """Pages full of tokens, as writing them leaves the pool: those behind a sequence's end hold what some other one left there."""
    nl, H, P = case["layers"], case["kv_heads"], case["page"]
    values = torch.empty((nl, n_pages, H, 2, P * HEAD_DIM), dtype=torch.uint8, device="cuda")
    exponents = torch.empty((nl, n_pages, H, 2), dtype=torch.int32, device="cuda")
    for layer in range(nl):
        for which in (0, 1):
            x = _normal((n_pages, H, P, HEAD_DIM), scale[layer][:, None, :] if which == 0 else None, torch.float32, gen)
            e = _exponent(x.abs().amax((2, 3)))
            x = _e4m3(_scaled(x, -e[:, :, None, None]))
            if which:
                x = x.view(n_pages, H, P // 8, 8, HEAD_DIM).transpose(3, 4)
            values[layer, :, :, which] = x.reshape(n_pages, H, P * HEAD_DIM)
            exponents[layer, :, :, which] = e
    return values, exponents


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens, news = _lengths(case)
    nl, H, P, B, dtype = case["layers"], case["kv_heads"], case["page"], case["batch"], _dtype(case)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    width = max(1, _pages(max(case["context"], 1), P)) + 2
    used = sum(_pages(n, P) for n in lens)
    base = [n - k for n, k in zip(lens, news)]
    if case["kind"] == "resize":
        at_first = sum(_pages(n, P) for n in base)
        n_pages = max(1, at_first, int(used * case["spare"]))
    else:
        at_first, n_pages = used, max(1, int(used * case["spare"]))
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    held = base if case["kind"] == "resize" else lens
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    count = ints([_pages(n, P) for n in held])
    mine = torch.arange(width, device="cuda")[None, :] < count[:, None]
    table[mine] = order[:at_first]
    starts = torch.cumsum(torch.cat([ints([0]), ints(news)]), 0).to(torch.int32)
    n_tokens = sum(news) + case["pad"]
    state = dict(case=case, table=table, lens=ints(held))
    if case["kind"] == "resize":
        free = torch.full((1 + n_pages,), -1, dtype=torch.int32, device="cuda")
        free[0] = n_pages - at_first
        free[1:1 + n_pages - at_first] = order[at_first:]
        state.update(free=free, base=ints(base), want=ints(lens), starts=torch.empty_like(starts), slots=ints([0] * n_tokens))
        _plain_resize(state["want"], table, state["lens"], free, state["starts"], state["slots"], P)  # the step before, which every pass takes back
        return state
    # K: log-uniform scales of the channels
    scale = 10.0 ** (2.0 * torch.rand((nl, H, HEAD_DIM), generator=gen, device="cuda") - 1.0)
    values, exponents = _pool(case, n_pages, scale, gen)
    state.update(values=values, exponents=exponents, longest=max(lens), most=max(news))
    if case["kind"] == "read":
        return state
    token = torch.arange(n_tokens, device="cuda")
    owner = torch.searchsorted(starts[1:].contiguous(), token, right=True).clamp_max(B - 1)
    position = ints(base)[owner] + token - starts[owner]
    if case["kind"] == "write":
        slots = table[owner, (position // P).clamp(0, width - 1)] * P + position % P
        state["slots"] = torch.where(token < starts[-1], slots, -1).to(torch.int32)
        louder = 2.0 ** (2.0 * torch.rand((1, n_tokens, 1, 1), generator=gen, device="cuda") - 1.0)  # some tokens outgrow their page's scale
        state["k"] = _normal((nl, n_tokens, H, HEAD_DIM), scale[:, None] * louder, dtype, gen)
        state["v"] = _normal((nl, n_tokens, H, HEAD_DIM), louder, dtype, gen)
        return state
    heads = H * case["group"]
    state.update(q=_normal((nl, n_tokens, heads, HEAD_DIM), None, dtype, gen), starts=starts,
                 out=torch.zeros((nl, n_tokens, heads, HEAD_DIM), dtype=dtype, device="cuda"))
    return state


# ------------------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _own(state)
    s, case = state, state["case"]
    P = case["page"]
    if case["kind"] == "resize":
        _plain_resize(s["base"], s["table"], s["lens"], s["free"], s["starts"], s["slots"], P)
        _plain_resize(s["want"], s["table"], s["lens"], s["free"], s["starts"], s["slots"], P)
        return {k: s[k] for k in ("table", "lens", "free", "starts", "slots")}
    if case["kind"] == "write":
        _plain_write(s["values"], s["exponents"], s["k"], s["v"], s["slots"], P)
        return {"values": s["values"].view(torch.float8_e4m3fn), "exponents": s["exponents"]}
    if case["kind"] == "read":
        K, V = _tokens(s["values"], s["exponents"], s["table"], s["lens"], s["longest"], P)
        return {"K": K.to(_dtype(case)), "V": V.to(_dtype(case))}
    _plain_attn(s["values"], s["exponents"], s["q"], s["starts"], s["table"], s["lens"], s["out"], s["longest"], s["most"], case)
    return s["out"]


def _own(s):
    from paper_2507_20030_amd import binding
    case = s["case"]
    layers, P = case["layers"], case["page"]
    if case["kind"] == "resize":  # the draft of a step taken back, the next one's pages
        for want in (s["base"], s["want"]):
            binding.iwdft_pages_resize(want, s["table"], s["lens"], s["free"], s["starts"], s["slots"], P)
        return {k: s[k] for k in ("table", "lens", "free", "starts", "slots")}
    if case["kind"] == "write":
        binding.iwdft_pages_write(s["values"], s["exponents"], s["k"], s["v"], s["slots"])
        return {"values": s["values"].view(torch.float8_e4m3fn), "exponents": s["exponents"]}
    if case["kind"] == "read":
        shape = (layers, case["batch"], case["kv_heads"], s["longest"], HEAD_DIM)
        K, V = (torch.empty(shape, dtype=_dtype(case), device="cuda") for _ in range(2))
        binding.iwdft_pages_read(s["values"], s["exponents"], s["table"], s["lens"], K, V)
        return {"K": K, "V": V}
    binding.iwdft_pages_attn(s["values"], s["exponents"], s["q"], s["starts"], s["table"], s["lens"], s["out"], n_sink=case["sink"],
                             n_recent=case["recent"])
    return s["out"]


# ------------------------------------------------------------------------------------------------------------------------ plain forms
def _exponent(amax):
    """Smallest e >= -100 with amax <= 448 * 2^e: 448 = 0.875 * 2^9."""
    m, k = torch.frexp(amax)
    e = k - 9 + (m > 0.875)
    return torch.where(amax > 0, e, LEAST_EXPONENT).clamp_min(LEAST_EXPONENT).to(torch.int32)


def _scaled(x, e):
    """x * 2^e in two exact powers, from their bits: the one that torch.ldexp computes is rounded."""
    half = torch.div(e, 2, rounding_mode="floor")
    return x * (half + 127 << 23).view(torch.float32) * (e - half + 127 << 23).view(torch.float32)


def _e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_resize(want, table, lens, free, starts, slots, P):
    B, W = table.shape
    n_pages, column = free.numel() - 1, torch.arange(W, device="cuda")[None, :]
    have = lens.long()
    want = torch.where(want < 0, have, want.long())
    down, up = want < have, (want > have) & (want <= W * P)
    had, get = _pages(have, P), _pages(want, P)
    gone = torch.where(down, had - get, 0)
    count, released = free[0].long(), gone.sum()
    need, new = torch.where(up, get - had, 0), torch.where(up, want - have, 0)
    up = up & (new.cumsum(0) <= slots.numel()) & ((need == 0) | (need.cumsum(0) <= count + released))
    need, new = torch.where(up, need, 0), torch.where(up, new, 0)
    to = torch.where(up | down, want, have)
    # what is given back, the last page of the last sequence first, goes on the stack; what is taken comes from its top
    leaves = (column >= get[:, None]) & (column < had[:, None]) & down[:, None]
    rank = released - leaves.flatten().cumsum(0)
    back = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda")
    back.scatter_(0, torch.where(leaves.flatten(), rank, n_pages), table.flatten())
    enters = (column >= had[:, None]) & (column < (had + need)[:, None])
    at = count + released - enters.flatten().cumsum(0)
    page = torch.where(at < count, free[1 + at.clamp(0, n_pages - 1)], back[(at - count).clamp(0, n_pages)])
    taken = need.sum()
    place = torch.arange(n_pages, device="cuda")
    free[1:] = torch.where((place >= count) & (place < count + released - taken), back[(place - count).clamp(0, n_pages)], free[1:])
    free[0] = count + released - taken
    table.copy_(torch.where(enters.flatten(), page, table.flatten()).view(B, W))
    lens.copy_(to)
    starts[0] = 0
    starts[1:] = new.cumsum(0)
    token = torch.arange(slots.numel(), device="cuda")
    owner = torch.searchsorted(starts[1:].long(), token, right=True).clamp_max(B - 1)
    position = have[owner] + token - starts[owner]
    slot = table[owner, (position // P).clamp(0, W - 1)] * P + position % P
    slots.copy_(torch.where(token < starts[-1], slot, -1))


def _plain_write(values, exponents, k, v, slots, P):
    nl, n_pages, H = exponents.shape[:3]
    K, V = values[:, :, :, 0].view(nl, n_pages, H, P, HEAD_DIM), values[:, :, :, 1].view(nl, n_pages, H, P // 8, HEAD_DIM, 8)
    there = slots >= 0
    at = torch.where(there, slots, n_pages * P).long()  # no slot: a page behind the last one, which is dropped
    page, offset = at // P, at % P
    first = torch.full((n_pages + 1,), P, device="cuda").scatter_reduce(0, page, offset, "amin")[:n_pages]  # of the page's tokens that are new
    old_token = torch.arange(P, device="cuda")[None, :] < torch.where(first < P, first, 0)[:, None]  # [page, token]
    for which, x in ((0, k), (1, v)):
        x = x.float()
        index = page[None, :, None].expand(nl, len(at), H)
        amax = torch.zeros((nl, n_pages + 1, H), device="cuda").scatter_reduce(1, index, x.abs().amax(3), "amax")[:, :n_pages]
        e_old = exponents[..., which]
        e_new = torch.maximum(_exponent(amax), torch.where(first[None, :, None] > 0, e_old, LEAST_EXPONENT))
        e_new = torch.where(first[None, :, None] < P, e_new, e_old)
        store = K if which == 0 else V.permute(0, 1, 2, 3, 5, 4).reshape(nl, n_pages, H, P, HEAD_DIM)
        grown = _scaled(store.view(torch.float8_e4m3fn).float(), (e_old - e_new)[..., None, None])
        keep = old_token[None, :, None, :, None]
        store = torch.where(keep, _e4m3(grown), store)
        fresh = _e4m3(_scaled(x, -e_new.gather(1, index.clamp_max(n_pages - 1))[..., None]))
        store = torch.cat([store.transpose(2, 3).reshape(nl, n_pages * P, H, HEAD_DIM), fresh[:, :1]], 1)
        store[:, at] = fresh
        store = store[:, :-1].view(nl, n_pages, P, H, HEAD_DIM).transpose(2, 3)
        if which == 0:
            K.copy_(store)
        else:
            V.copy_(store.reshape(nl, n_pages, H, P // 8, 8, HEAD_DIM).transpose(4, 5))
        exponents[..., which] = e_new


def _tokens(values, exponents, table, lens, n, P):
    """K, V of the first n tokens, 0 where a sequence has fewer: fp32 [layers, sequences, KV heads, n, 128]."""
    nl, n_pages, H = exponents.shape[:3]
    B, got = table.shape[0], []
    token = torch.arange(n, device="cuda")
    page = table[:, token // P].long().clamp(0, n_pages - 1)  # [sequence, token]
    there = (token[None, :] < lens[:, None])[None, :, None, :, None]
    for which in (0, 1):
        store = values[:, :, :, which]
        store = store.view(nl, n_pages, H, P, HEAD_DIM) if which == 0 else store.view(nl, n_pages, H, P // 8, HEAD_DIM, 8).transpose(4, 5).reshape(
            nl, n_pages, H, P, HEAD_DIM)
        x = store.view(torch.uint8)[:, page, :, token % P].view(torch.float8_e4m3fn)  # the two indices apart: [sequence, token] leads
        x = x.permute(2, 0, 3, 1, 4).float()
        e = exponents[..., which][:, page].transpose(2, 3)[..., None]
        got.append(torch.where(there, _scaled(x, e), 0.0))
    return got


def _plain_attn(values, exponents, q, starts, table, lens, out, longest, most, case):
    nl, n_tokens, heads = q.shape[:3]
    B, H, P = table.shape[0], exponents.shape[2], case["page"]
    G = heads // H
    K, V = _tokens(values, exponents, table, lens, longest, P)
    new = starts[1:] - starts[:-1]
    row, column = torch.arange(most, device="cuda"), torch.arange(longest, device="cuda")
    pick = (starts[:-1, None] + row[None, :]).clamp_max(n_tokens - 1).long()  # [sequence, its new tokens]
    x = q.float()[:, pick].view(nl, B, most, H, G, HEAD_DIM).permute(0, 1, 3, 4, 2, 5).reshape(nl, B, H, G * most, HEAD_DIM)
    scores = torch.matmul(x, K.transpose(3, 4).contiguous()).view(nl, B, H, G, most, longest)
    scores *= HEAD_DIM ** -0.5
    position = (lens[:, None] - new[:, None] + row[None, :])[:, :, None]  # [sequence, new token, 1]
    visible = column <= position
    if case["recent"]:
        visible &= (column < case["sink"]) | (column > position - case["recent"])
    visible = visible[None, :, None, None]
    scores.masked_fill_(~visible, -math.inf)
    scores -= scores.amax(5, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    scores.exp_()
    total = scores.sum(5, keepdim=True)
    y = torch.matmul(scores.view(nl, B, H, G * most, longest), V).view(nl, B, H, G, most, HEAD_DIM)
    y = torch.where(total > 0, y / total, 0.0).permute(0, 1, 4, 2, 3, 5).reshape(nl, B, most, heads, HEAD_DIM)
    token = torch.arange(n_tokens, device="cuda")
    owner = torch.searchsorted(starts[1:].contiguous(), token, right=True).clamp_max(B - 1)
    mine = y[:, owner, (token - starts[owner]).clamp(0, most - 1)].to(out.dtype)
    out.copy_(torch.where((token < starts[-1])[None, :, None, None], mine, out))


# -------------------------------------------------------------------------------------------------------------------- work, definition
def work(case):
    lens, news = _lengths(case)
    P, H, G, nl, item = case["page"], case["kv_heads"], case["group"], case["layers"], _dtype(case).itemsize
    tokens, new = sum(lens), sum(news)
    if case["kind"] == "resize":
        entries = sum(_pages(n, P) - _pages(n - k, P) for n, k in zip(lens, news))
        # back: entries read and pushed; forth: popped and entered; slots, lengths, wanted lengths, starts of both calls
        return dict(bytes=4 * (4 * entries + 2 * (new + case["pad"]) + 8 * case["batch"]), flops=0)
    cells = nl * H * HEAD_DIM * 2  # of one token, K and V
    if case["kind"] == "write":
        return dict(bytes=cells * new * (item + 1) + 4 * (new + case["pad"]), flops=2 * cells * new)
    if case["kind"] == "read":
        return dict(bytes=cells * (tokens + case["batch"] * max(lens) * item), flops=cells * tokens)
    pairs, read = 0, 0
    for n, k in zip(lens, news):
        counts = _visible_counts(n, k, case["sink"], case["recent"])
        pairs += counts[0]
        read += counts[1] if k else 0
    return dict(bytes=cells * read + 2 * nl * new * H * G * HEAD_DIM * item, flops=4 * HEAD_DIM * nl * H * G * pairs)


def _visible_counts(n, k, sink, recent):
    """(pairs of a new token and a token that it sees, tokens that some new token sees) of a sequence of n tokens, k of them new."""
    if not recent:
        return k * n - k * (k - 1) // 2, n
    pairs = 0
    for p in range(n - k, n):
        near = min(recent, p + 1)
        pairs += near + min(sink, p + 1 - near)
    near = min(n, recent + max(0, k - 1))
    return pairs, near + min(sink, n - near)


def _grid_values():
    """What the 256 bytes of e4m3 stand for."""
    got = []
    for byte in range(256):
        e, m = byte >> 3 & 15, byte & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v = math.nan if byte & 127 == 127 else v
        got.append(-v if byte & 128 else v)
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _power(e):
    return torch.tensor([2.0 ** k for k in range(-300, 300)], dtype=torch.float64, device="cuda")[e.long() + 300]


def _exact_store(state, layer, which):
    """One layer's K or V as stored, 64 bits: (values [pages, heads, P, 128], exponents [pages, heads])."""
    P = state["case"]["page"]
    raw = _grid_values()[state["values"][layer, :, :, which].int()]
    n, h = raw.shape[:2]
    raw = raw.view(n, h, P, HEAD_DIM) if which == 0 else raw.view(n, h, P // 8, HEAD_DIM, 8).permute(0, 1, 2, 4, 3).reshape(n, h, P, HEAD_DIM)
    return raw, state["exponents"][layer, :, :, which]


def exact(case, seed):
    if case["kind"] == "resize":
        return None
    state = prepare(case, seed)
    P, nl, (lens, news) = case["page"], case["layers"], _lengths(case)
    if case["kind"] == "write":
        return {"values": _exact_write(state, P), "exponents": None}
    table = state["table"].tolist()
    base = [sum(news[:b]) for b in range(len(news))]
    if case["kind"] == "read":
        got = torch.zeros((2, nl, case["batch"], case["kv_heads"], max(lens), HEAD_DIM), dtype=torch.float64, device="cuda")
    else:
        got = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    for layer in range(nl):
        (kv, ke), (vv, ve) = (_exact_store(state, layer, w) for w in (0, 1))
        for b, n in enumerate(lens):
            if not n:
                continue
            pages = torch.tensor(table[b][:_pages(n, P)], device="cuda")
            k, v = ((x[pages] * _power(e[pages])[:, :, None, None]).transpose(0, 1).reshape(case["kv_heads"], -1, HEAD_DIM)[:, :n]
                    for x, e in ((kv, ke), (vv, ve)))
            if case["kind"] == "read":
                got[0, layer, b, :, :n], got[1, layer, b, :, :n] = k, v
                continue
            rows = slice(base[b], base[b] + news[b])
            p, j = torch.arange(n - news[b], n, device="cuda")[:, None], torch.arange(n, device="cuda")[None, :]
            hidden = j > p
            if case["recent"]:
                hidden = hidden | ((j >= case["sink"]) & (j <= p - case["recent"]))
            for head in range(case["kv_heads"] * case["group"] if news[b] else 0):
                h = head // case["group"]
                s = state["q"][layer, rows, head].double() @ k[h].T / math.sqrt(HEAD_DIM)
                got[layer, rows, head] = torch.softmax(s.masked_fill_(hidden, -math.inf), dim=1) @ v[h]
    return {"K": got[0], "V": got[1]} if case["kind"] == "read" else got


def _exact_write(state, P):
    """The pool's numbers after the write, from the definition: exponent by comparison with powers of two, rounding on the grid in 64 bits."""
    slots = state["slots"].tolist()
    rows = {}
    for t, s in enumerate(slots):
        if s >= 0:
            rows.setdefault(s // P, []).append((s % P, t))
    power = 448.0 * _power(torch.arange(LEAST_EXPONENT, 121, device="cuda"))
    pages = torch.tensor(sorted(rows), device="cuda")
    first = torch.tensor([rows[p][0][0] for p in sorted(rows)], device="cuda")
    token = torch.full((len(rows), P), -1)
    for i, p in enumerate(sorted(rows)):
        for offset, t in rows[p]:
            token[i, offset] = t
    token = token.cuda()
    out = torch.empty(state["values"].shape, dtype=torch.float64, device="cuda")
    for layer in range(out.shape[0]):
        for which, name in ((0, "k"), (1, "v")):
            stored, e = _exact_store(state, layer, which)
            x = state[name][layer].double()[token.clamp_min(0)].transpose(1, 2)  # [page, head, P, 128]
            new = (token >= 0)[:, None, :, None]
            amax = torch.where(new, x.abs(), 0.0).amax((2, 3))
            up = torch.searchsorted(power, amax) + LEAST_EXPONENT
            old = e[pages].long()
            up = torch.where((first > 0)[:, None], torch.maximum(up, old), up)
            kept = torch.arange(P, device="cuda")[None, :] < first[:, None]
            moved = _round_e4m3(stored[pages] * _power(old - up)[:, :, None, None])
            page = torch.where(kept[:, None, :, None], moved, stored[pages])
            page = torch.where(new, _round_e4m3(x * _power(-up)[:, :, None, None]), page)
            stored[pages] = page
            if which:
                n, h = stored.shape[:2]
                stored = stored.view(n, h, P // 8, 8, HEAD_DIM).transpose(3, 4)
            out[layer, :, :, which] = stored.reshape(stored.shape[0], stored.shape[1], -1)
    return out


def _round_e4m3(x):
    """Nearest number of the grid, ties to even: three bits behind the leading one, steps of 2^-9 below 2^-6."""
    step = _power(torch.frexp(x.abs().clamp_min(2.0 ** -6))[1] - 4)
    return torch.round(x / step) * step
