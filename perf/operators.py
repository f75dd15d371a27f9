"""The operators of a verification step beside its products, as cases that can be timed and compared.

  slots      block tables and slot maps from request lengths (`kv_slots`)
  append     keys and values of new tokens into a paged cache (`kv_append`)
  attention  the drafted tokens of every request, a tree each, over its cached context (`tree_attention`)
  adapters   low-rank adapters of many requests beside a shared projection (`lora_smallm`)
  rules      penalties for repeated tokens, biases and grammar masks on logits (`logits_rules`)

`run` computes them with elementary torch operations, or, where `own` is true, through the public calls of
`paper_2605_11582_amd.binding`.  Every request of a batch has another length: the lengths are spread evenly over their
range and dealt to the requests by the seed, so that the work of a case does not depend on it.
"""
import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # a verification step of 48 requests with up to 16 accepted tokens each, pages of 16: latency counts
        {"name": "slots_step", "op": "slots", "requests": 48, "most": 16, "context": 8192, "page": 16, "short": False},
        # prompts of 512 requests enter the cache at once, and its free pages do not suffice for all of them
        {"name": "slots_prompts", "op": "slots", "requests": 512, "most": 2048, "context": 4096, "page": 64, "short": True},
        # the accepted tokens of a step: 64 entries, some of them rejected, rows picked from the drafted ones
        {"name": "append_step", "op": "append", "tokens": 64, "heads": 8, "dim": 128, "page": 16, "slots": 16384, "picked": True, "by_token": False},
        # 16384 tokens of prompts, 32 heads, pages laid out token by token
        {"name": "append_prompts", "op": "append", "tokens": 16384, "heads": 32, "dim": 128, "page": 64, "slots": 24576, "picked": False, "by_token": True},
        # one token of one request over a short context: the smallest decoding step of a 4096-wide decoder
        {"name": "attention_one", "op": "attention", "requests": 1, "tokens": 1, "context": 777, "heads": 32, "kv_heads": 32, "dim": 128, "page": 16, "by_token": False},
        # sixteen requests with up to 20 candidates each (the beam width of the targeted-advertising setting), shared heads
        {"name": "attention_beam", "op": "attention", "requests": 16, "tokens": 20, "context": 4096, "heads": 32, "kv_heads": 8, "dim": 128, "page": 32, "by_token": False},
        # the most candidates a request may have over a long context (the largest)
        {"name": "attention_long", "op": "attention", "requests": 1, "tokens": 64, "context": 131072, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "by_token": False},
        # heads of 80, seven query heads a key head, short pages laid out token by token, an empty context among them
        {"name": "attention_odd", "op": "attention", "requests": 7, "tokens": 33, "context": 3001, "heads": 14, "kv_heads": 2, "dim": 80, "page": 8, "by_token": True},
        # sixteen tokens of a step, four adapters of rank 16 beside a 4096 x 4096 projection
        {"name": "adapters_16_4096x4096", "op": "adapters", "tokens": 16, "cols": 4096, "rows": 4096, "rank": 16, "adapters": 4},
        # 64 tokens that use most of 64 adapters of rank 32 beside the gate projection
        {"name": "adapters_64_11008x4096", "op": "adapters", "tokens": 64, "cols": 4096, "rows": 11008, "rank": 32, "adapters": 64},
        # one row of an odd vocabulary: a single decoding step
        {"name": "rules_one", "op": "rules", "requests": 1, "tokens": 1, "vocab": 32003, "history": 600, "kind": "fp16", "masks": 1},
        # the candidates of sixteen requests, up to eight each, long histories
        {"name": "rules_candidates", "op": "rules", "requests": 16, "tokens": 8, "vocab": 128000, "history": 4096, "kind": "fp16", "masks": 40},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["slots", "append", "attention", "attention", "attention", "adapters", "adapters", "rules"])
    if op == "slots":
        requests = _log(rng, 1, 1024)
        return {"op": op, "requests": requests, "most": _log(rng, 1, min(4096, (1 << 20) // requests)), "context": _log(rng, 16, 16384),
                "page": rng.choice([1, 8, 16, 32, 64, 128]), "short": rng.random() < 0.3}
    if op == "append":
        tokens = _log(rng, 1, 16384)
        return {"op": op, "tokens": tokens, "heads": rng.choice([1, 2, 5, 8, 8, 16, 32]), "dim": rng.choice([32, 64, 80, 96, 128, 128, 256]),
                "page": rng.choice([1, 8, 16, 32, 64]), "slots": tokens + _log(rng, 64, 8192), "picked": rng.random() < 0.5, "by_token": rng.random() < 0.5}
    if op == "attention":
        requests = _log(rng, 1, 64)
        kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 256])
        context = _log(rng, 16, min(131072, (1 << 26) // (requests * kv_heads * dim)))
        shared = rng.choice([1, 1, 2, 3, 4, 7, 8])
        # (the plain form's scores in 32 bits are held to a gigabyte)
        tokens = _log(rng, 1, max(1, min(64, (1 << 28) // (requests * kv_heads * shared * context))))
        return {"op": op, "requests": requests, "tokens": tokens, "context": context, "heads": kv_heads * shared, "kv_heads": kv_heads, "dim": dim,
                "page": rng.choice([1, 8, 16, 16, 32, 64, 128]), "by_token": rng.random() < 0.4}
    if op == "adapters":
        rank, cols = 8 * rng.choice([1, 2, 2, 4, 4, 5, 8, 16]), 32 * _log(rng, 16, 400)
        rows = _log(rng, 500, 14000)
        tokens = _log(rng, 1, 64)
        return {"op": op, "tokens": tokens, "cols": cols, "rows": rows, "rank": rank, "adapters": _log(rng, 1, max(1, min(128, (1 << 28) // (rank * (cols + rows)))))}
    requests, tokens = _log(rng, 1, 32), _log(rng, 1, 64)
    return {"op": op, "requests": requests, "tokens": tokens, "vocab": _log(rng, 1000, min(200000, (1 << 24) // (requests * tokens))), "history": _log(rng, 1, 8192),
            "kind": rng.choice(["fp16", "fp16", "fp32"]), "masks": rng.choice([0, 1, 5, 32])}


# ---------------------------------------------------------------- inputs
def _spread(order, lo, hi):
    """Whole numbers from lo to hi, one for each request, in the given order; hi for a single request."""
    n = len(order)
    return np.array([hi if n == 1 else lo + (hi - lo) * k // (n - 1) for k in order], dtype=np.int32)


def _int(a, kind=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=kind)).cuda()


def _trees(rs, counts):
    """Which drafted tokens a token sees, as bits: itself and its ancestors in a random tree of its request."""
    words = []
    for c in counts:
        seen = []
        for j in range(c):
            parent = rs.randint(-1, j) if j else -1          # (-1: hangs on the context itself)
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << j)
        words += seen
    return np.array(words, dtype=np.uint64).view(np.int64)


def _cache(gen, case, blocks):
    """Keys or values as (blocks, heads, page, dim), the tokens or the heads of a page outermost in memory."""
    page, heads, dim = case["page"], case.get("kv_heads", case["heads"]), case["dim"]
    if case["by_token"]:
        return torch.randn((blocks, page, heads, dim), generator=gen, device="cuda", dtype=torch.float16).transpose(1, 2)
    return torch.randn((blocks, heads, page, dim), generator=gen, device="cuda", dtype=torch.float16)


def _slots_numbers(case):
    return -(-(case["context"] + case["most"]) // case["page"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))
    op = case["op"]
    state = {"case": case}
    if op == "slots":
        n, page = case["requests"], case["page"]
        width = _slots_numbers(case)
        lens, counts = _spread(rs.permutation(n), 0, case["context"]), _spread(rs.permutation(n), 0, case["most"])
        have = -(-lens // page)
        need = -(-(lens + counts) // page) - have
        blocks = n * width + 7
        ids = rs.permutation(blocks).astype(np.int32)
        table = np.where(np.arange(width) < have[:, None], ids[:n * width].reshape(n, width), -1)
        free = np.concatenate([ids[:n * width].reshape(n, width)[np.arange(width) >= have[:, None]], ids[n * width:]])
        head = 3
        if case["short"]:
            free = free[:head + int(need.sum()) // 2]
        state.update(lens=_int(lens), counts=_int(counts), table=_int(table), free=_int(free), head=_int([head]), blocks=blocks,
                     slots=torch.zeros(n * case["most"], dtype=torch.int32, device="cuda"), cu=torch.zeros(n + 1, dtype=torch.int32, device="cuda"),
                     new_lens=torch.zeros(n, dtype=torch.int32, device="cuda"), new_head=torch.zeros(1, dtype=torch.int32, device="cuda"))
    elif op == "append":
        n, heads, dim = case["tokens"], case["heads"], case["dim"]
        blocks = -(-case["slots"] // case["page"])
        kv = torch.randn((n, 2 * heads, dim), generator=gen, device="cuda", dtype=torch.float16)    # one projection's output
        slots = rs.permutation(blocks * case["page"])[:n]
        slots[rs.rand(n) < 0.2] = -1                          # rejected candidates, padding
        state.update(k=kv[:, :heads], v=kv[:, heads:], k_cache=_cache(gen, case, blocks), v_cache=_cache(gen, case, blocks), slots=_int(slots),
                     rows=_int(rs.permutation(n)) if case["picked"] else None)
    elif op == "attention":
        n, most, page, heads, kv_heads, dim = (case[k] for k in ("requests", "tokens", "page", "heads", "kv_heads", "dim"))
        lens, counts = _spread(rs.permutation(n), 0, case["context"]), _spread(rs.permutation(n), 1, most)
        width = -(-case["context"] // page)
        cu = np.concatenate([[0], np.cumsum(counts)])
        mask = np.zeros(n * most, dtype=np.int64)
        mask[:cu[-1]] = _trees(rs, counts)
        qkv = torch.randn((n * most, heads + 2 * kv_heads, dim), generator=gen, device="cuda", dtype=torch.float16)
        state.update(q=qkv[:, :heads], k=qkv[:, heads:heads + kv_heads], v=qkv[:, heads + kv_heads:], k_cache=_cache(gen, case, n * width),
                     v_cache=_cache(gen, case, n * width), table=_int(rs.permutation(n * width).reshape(n, width)), lens=_int(lens), cu=_int(cu),
                     mask=_int(mask, np.int64), out=torch.zeros((n * most, heads, dim), dtype=torch.float16, device="cuda"), scale=dim ** -0.5)
    elif op == "adapters":
        m, cols, rows, rank, n = (case[k] for k in ("tokens", "cols", "rows", "rank", "adapters"))
        index = rs.randint(0, n, m)
        index[rs.rand(m) < 0.1] = -1                          # requests without an adapter
        state.update(x=torch.randn((m, cols), generator=gen, device="cuda", dtype=torch.float16),
                     a=torch.randn((n, rank, cols), generator=gen, device="cuda", dtype=torch.float16) * 0.02,
                     b=torch.randn((n, rows, rank), generator=gen, device="cuda", dtype=torch.float16) * 0.02,
                     base=torch.randn((m, rows), generator=gen, device="cuda", dtype=torch.float16), index=_int(index),
                     factor=torch.rand(n, generator=gen, device="cuda") * 2 + 0.25, y=torch.zeros((m, rows), dtype=torch.float16, device="cuda"))
    else:
        n, most, vocab, length = case["requests"], case["tokens"], case["vocab"], case["history"]
        counts, lens = _spread(rs.permutation(n), 1, most), _spread(rs.permutation(n), 0, length)
        cu = np.concatenate([[0], np.cumsum(counts)])
        mask = np.zeros(n * most, dtype=np.int64)
        mask[:cu[-1]] = _trees(rs, counts)
        ids = (vocab * rs.rand(n, length) ** 3).astype(np.int32)                   # frequent words repeat
        bias_ids = (vocab * rs.rand(n, 24)).astype(np.int32)
        bias_ids[rs.rand(n, 24) < 0.3] = -1
        bias_ids[:, 3] = bias_ids[:, 11]                      # an id named twice
        logits = torch.randn((n * most, vocab), generator=gen, device="cuda", dtype=torch.float32) * 4
        masks = case["masks"]
        state.update(logits=logits.to(torch.float16 if case["kind"] == "fp16" else torch.float32), cu=_int(cu), history=_int(ids), history_len=_int(lens),
                     prompt_len=_int(lens // 3), draft=_int((vocab * rs.rand(n * most) ** 3)), mask=_int(mask, np.int64),
                     repetition=torch.rand(n, generator=gen, device="cuda") * 0.5 + 1, frequency=torch.rand(n, generator=gen, device="cuda"),
                     presence=torch.rand(n, generator=gen, device="cuda"), bias_ids=_int(bias_ids), bias=torch.randn((n, 24), generator=gen, device="cuda") * 3,
                     allowed=torch.randint(-(1 << 31), 1 << 31, (masks, -(-vocab // 32)), generator=gen, device="cuda", dtype=torch.int32) if masks else None,
                     allowed_row=_int(rs.randint(-1, masks, n * most)) if masks else None)
        state["out"] = torch.zeros_like(state["logits"])
    return state


# ---------------------------------------------------------------- one pass: plain forms
def _requests_of(cu, rows):
    """The request of every row of a batch; rows past the last request get the number of requests."""
    return torch.searchsorted(cu[1:], torch.arange(rows, device=cu.device, dtype=cu.dtype), right=True)


def _plain_slots(s):
    page, lens, counts, table, free, head = s["case"]["page"], s["lens"].long(), s["counts"].long(), s["table"].long(), s["free"].long(), s["head"].long()
    n, width, capacity = *table.shape, s["slots"].numel()
    have = -(-lens // page)
    ends = counts.cumsum(0)
    cu = torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=capacity)
    room = (lens + counts <= width * page) & (ends <= capacity)
    need = torch.where(room, -(-(lens + counts) // page) - have, 0)
    upto = need.cumsum(0)
    start = upto - need
    kept = room & ((need == 0) | (upto <= free.numel() - head))
    new_head = head + torch.where(kept & (need > 0), upto, 0).max()
    col = torch.arange(width, device=lens.device) - have[:, None]
    taken = free[(head + start[:, None] + col).clamp(0, free.numel() - 1)]
    table = torch.where(kept[:, None] & (col >= 0) & (col < need[:, None]), taken, table)
    i = torch.arange(capacity, device=lens.device)
    b = _requests_of(cu, capacity)
    at = b.clamp(max=n - 1)
    pos = lens[at] + i - cu[at]
    block = table.view(-1)[(at * width + (pos // page).clamp(0, width - 1))]
    slots = torch.where((b < n) & kept[at] & (block >= 0) & (block < s["blocks"]), block * page + pos % page, -1)
    return [t.to(torch.int32) for t in (slots, cu, torch.where(kept, lens + counts, lens), new_head, table)]


def _plain_append(s):
    slots, rows = s["slots"].long(), s["rows"]
    page = s["case"]["page"]
    rows = torch.arange(slots.numel(), device=slots.device) if rows is None else rows.long()
    fine = slots >= 0
    one = fine.to(torch.int32).argmax()                       # entries without a slot repeat this one
    slots, rows = torch.where(fine, slots, slots[one].clamp(min=0)), torch.where(fine, rows, rows[one])
    for new, cache in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
        at = (slots // page, slice(None), slots % page)
        cache[at] = torch.where(fine.any(), new[rows], cache[at])
    return s["k_cache"], s["v_cache"]


def _plain_attention(s):
    q, k, v, cu, lens = s["q"], s["k"], s["v"], s["cu"].long(), s["lens"].long()
    (rows, heads, dim), kv_heads, n, most, page = q.shape, k.shape[1], lens.numel(), s["case"]["tokens"], s["case"]["page"]
    shared, width = heads // kv_heads, s["table"].shape[1] * page
    token = torch.arange(most, device=q.device)
    counts = cu[1:] - cu[:-1]
    at = (cu[:-1, None] + token).clamp(max=rows - 1)          # (requests, tokens): their rows
    # keys and values of a request one after the other: its pages, then its drafted tokens
    def whole(cache, new):
        pages = cache[s["table"].long()].permute(0, 2, 1, 3, 4).reshape(n, kv_heads, width, dim)
        return torch.cat([pages, new[at].transpose(1, 2)], 2).float()
    bit = (s["mask"][at][:, :, None] >> token) & 1 == 1
    seen = torch.cat([(torch.arange(width, device=q.device) < lens[:, None])[:, None, :].expand(-1, most, -1), bit & (token < counts[:, None])[:, None, :]], 2)
    seen = seen[:, None, None]                                # (requests, 1, 1, tokens, keys)
    qs = q[at].view(n, most, kv_heads, shared, dim).permute(0, 2, 3, 1, 4).float()
    keys, values = whole(s["k_cache"], k), whole(s["v_cache"], v)
    scores = (qs.reshape(n, kv_heads, shared * most, dim) @ keys.transpose(2, 3)).view(n, kv_heads, shared, most, -1) * s["scale"]
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(4, keepdim=True)
    weight = scores.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = weight.sum(4, keepdim=True)
    o = (weight.view(n, kv_heads, shared * most, -1) @ values).view(n, kv_heads, shared, most, dim) / torch.where(total == 0, 1, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(n * most, heads, dim)
    b = _requests_of(cu, rows)
    i = torch.arange(rows, device=q.device)
    mine = b.clamp(max=n - 1)
    return torch.where((b < n)[:, None, None], o[mine * most + (i - cu[mine]).clamp(0, most - 1)].half(), s["out"])


def _plain_adapters(s):
    index = s["index"].long()
    one = index.clamp(min=0)
    h = s["a"][one].float() @ s["x"].float()[:, :, None]
    change = (s["b"][one].float() @ h)[:, :, 0] * s["factor"][one][:, None]
    return (s["base"].float() + torch.where(index[:, None] >= 0, change, 0)).half()


def _plain_rules(s):
    logits, cu = s["logits"], s["cu"].long()
    (rows, vocab), (n, length), most = logits.shape, s["history"].shape, s["case"]["tokens"]
    device = logits.device
    b = _requests_of(cu, rows)
    used, mine = b < n, b.clamp(max=n - 1)
    place = torch.arange(length, device=device)
    written = (place < s["history_len"][:, None]) & (place >= s["prompt_len"][:, None])
    prompt = place < torch.minimum(s["prompt_len"], s["history_len"])[:, None]
    ids = s["history"].long()
    count = torch.zeros((n, vocab), device=device).scatter_add_(1, ids, written.float())[mine]
    told = torch.zeros((n, vocab), device=device).scatter_add_(1, ids, prompt.float())[mine] > 0
    # the drafted tokens that a row sees count as written
    token = torch.arange(most, device=device)
    drafted = s["draft"].long()[(cu[mine][:, None] + token).clamp(max=rows - 1)]
    sees = ((s["mask"][:, None] >> token) & 1 == 1) & (token < (cu[mine + 1] - cu[mine])[:, None])
    count = count.scatter_add_(1, drafted, sees.float())
    per = lambda t: t[mine][:, None]  # noqa: E731
    x = logits.float()
    x = torch.where(told | (count > 0), torch.where(x > 0, x / per(s["repetition"]), x * per(s["repetition"])), x)
    x = x - per(s["frequency"]) * count - torch.where(count > 0, per(s["presence"]), 0)
    # of an id that is named twice the last entry counts
    which = s["bias_ids"].long()
    entry = torch.arange(which.shape[1], device=device).expand_as(which)
    last = torch.full((n, vocab + 1), -1, device=device).scatter_reduce_(1, torch.where(which < 0, vocab, which), entry, "amax")[mine, :vocab]
    x = x + torch.where(last >= 0, s["bias"][mine].gather(1, last.clamp(min=0)), 0)
    if s["allowed"] is not None:
        v = torch.arange(vocab, device=device)
        row = s["allowed_row"].long()
        bits = (s["allowed"][row.clamp(min=0)][:, v // 32] >> (v % 32).int()) & 1 == 1
        x = torch.where(bits | (row < 0)[:, None], x, -math.inf)
    return torch.where(used[:, None], x.to(logits.dtype), s["out"])


# ---------------------------------------------------------------- one pass
def run(state):
    s, op = state, state["case"]["op"]
    if own:
        from paper_2605_11582_amd import binding as egt
        if op == "slots":
            egt.kv_slots(s["lens"], s["counts"], s["table"], s["case"]["page"], s["blocks"], s["free"], s["head"], s["slots"], s["cu"], s["new_lens"], s["new_head"])
            return [s["slots"], s["cu"], s["new_lens"], s["new_head"], s["table"]]
        if op == "append":
            egt.kv_append(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"], rows=s["rows"])
            return s["k_cache"], s["v_cache"]
        if op == "attention":
            if "workspace" not in s:                          # (made once, as a serving program does)
                need = egt.tree_attention_ws_bytes(s["q"], s["k_cache"], s["table"], s["lens"], s["case"]["tokens"])
                s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
            egt.tree_attention(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["cu"], s["mask"], s["out"], s["scale"],
                               s["case"]["tokens"], s["workspace"])
            return s["out"]
        if op == "adapters":
            if "workspace" not in s:
                s["workspace"] = torch.empty(egt.lora_smallm_ws_bytes(s["x"], s["a"]), dtype=torch.uint8, device="cuda")
            egt.lora_smallm(s["x"], s["a"], s["b"], s["index"], s["y"], s["workspace"], base=s["base"], scale=s["factor"])
            return s["y"]
        egt.logits_rules(s["logits"], s["out"], s["cu"], history=s["history"], history_len=s["history_len"], prompt_len=s["prompt_len"], draft=s["draft"],
                         mask=s["mask"], repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"], bias_ids=s["bias_ids"], bias=s["bias"],
                         allowed=s["allowed"], allowed_row=s["allowed_row"])
        return s["out"]
    return {"slots": _plain_slots, "append": _plain_append, "attention": _plain_attention, "adapters": _plain_adapters, "rules": _plain_rules}[op](s)


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "slots":
        return None                                           # whole numbers
    if op == "append":
        for new, cache in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
            src = new if s["rows"] is None else new.index_select(0, s["rows"])
            for which, block, off in zip(*[t.tolist() for t in (torch.nonzero(s["slots"] >= 0)[:, 0], *torch.unravel_index(s["slots"][s["slots"] >= 0], (cache.shape[0], case["page"])))]):
                cache[block, :, off] = src[which]
        return s["k_cache"].double(), s["v_cache"].double()
    if op == "attention":
        out = s["out"].double()
        cu, lens = s["cu"].tolist(), s["lens"].tolist()
        group = case["heads"] // case["kv_heads"]
        for r in range(case["requests"]):
            first, last = cu[r], cu[r + 1]
            words = s["mask"][first:last].tolist()
            sight = torch.tensor([[(w >> j) & 1 for j in range(last - first)] for w in words], dtype=torch.bool, device="cuda")
            pages = s["table"][r, :-(-lens[r] // case["page"])].long()
            for h in range(case["kv_heads"]):
                old = [c[pages, h].reshape(-1, case["dim"])[:lens[r]] for c in (s["k_cache"], s["v_cache"])]
                keys, values = (torch.cat([a, b[first:last, h]]).double() for a, b in zip(old, (s["k"], s["v"])))
                for g in range(group):
                    e = s["q"][first:last, h * group + g].double() @ keys.T / math.sqrt(case["dim"])
                    e[:, lens[r]:][~sight] = -math.inf
                    out[first:last, h * group + g] = torch.softmax(e, 1) @ values
        return out
    if op == "adapters":
        out = s["base"].double()
        for m, a in enumerate(s["index"].tolist()):
            if a >= 0:
                out[m] += s["factor"][a].double() * torch.mv(s["b"][a].double(), torch.mv(s["a"][a].double(), s["x"][m].double()))
        return out
    out = s["out"].double()
    cu, hist, lens, prompts = (s[k].tolist() for k in ("cu", "history", "history_len", "prompt_len"))
    draft, words, names, bias = (s[k].tolist() for k in ("draft", "mask", "bias_ids", "bias"))
    for r in range(case["requests"]):
        base_count = np.bincount(hist[r][prompts[r]:lens[r]], minlength=case["vocab"]).astype(np.float64)
        prompt = np.bincount(hist[r][:prompts[r]], minlength=case["vocab"]) > 0
        theta, alpha, beta = (float(s[k][r].double()) for k in ("repetition", "frequency", "presence"))
        add = np.zeros(case["vocab"])
        for t, v in zip(names[r], bias[r]):
            if t >= 0:
                add[t] = v
        for i in range(cu[r], cu[r + 1]):
            count = base_count.copy()
            for j in range(cu[r + 1] - cu[r]):
                count[draft[cu[r] + j]] += (words[i] >> j) & 1
            x = s["logits"][i].double().cpu().numpy()
            x = np.where(prompt | (count > 0), np.where(x > 0, x / theta, x * theta), x) - alpha * count - beta * (count > 0) + add
            if case["masks"] and (row := int(s["allowed_row"][i])) >= 0:
                bits = np.unpackbits(s["allowed"][row].cpu().numpy().view(np.uint8), bitorder="little")[:case["vocab"]]
                x[bits == 0] = -np.inf
            out[i] = torch.from_numpy(x).cuda()
    return out


# ---------------------------------------------------------------- what a pass cannot do without
def _total(n, lo, hi):
    return int(_spread(range(n), lo, hi).sum())


def work(case):
    op = case["op"]
    if op == "slots":
        n, tokens = case["requests"], _total(case["requests"], 0, case["most"])
        # lengths and counts in, lengths and offsets out, every slot, every page that is taken (read and written)
        return {"bytes": 16 * n + 4 * n * case["most"] + 8 * (tokens // case["page"]), "flops": 0}
    if op == "append":
        return {"bytes": case["tokens"] * (4 + 8 * case["heads"] * case["dim"]), "flops": 0}
    if op == "attention":
        n, heads, kv_heads, dim = case["requests"], case["heads"], case["kv_heads"], case["dim"]
        context, tokens = _total(n, 0, case["context"]), _total(n, 1, case["tokens"])
        keys = context + tokens
        # (every token meets its request's context: the mean of one times the mean of the other)
        return {"bytes": 4 * keys * kv_heads * dim + 4 * tokens * heads * dim + 4 * context // case["page"],
                "flops": 4 * heads * dim * tokens * keys // n}
    if op == "adapters":
        m, cols, rows, rank, n = (case[k] for k in ("tokens", "cols", "rows", "rank", "adapters"))
        used = n * (1 - (1 - 1 / n) ** (0.9 * m))             # adapters that some token has, on average
        return {"bytes": int(2 * used * rank * (cols + rows)) + 2 * m * (cols + 2 * rows), "flops": int(1.8 * m * rank * (cols + rows))}
    n, rows, vocab = case["requests"], _total(case["requests"], 1, case["tokens"]), case["vocab"]
    masks = min(case["masks"], rows) * vocab // 8
    return {"bytes": (4 if case["kind"] == "fp16" else 8) * rows * vocab + masks + 4 * _total(n, 0, case["history"]), "flops": 4 * rows * vocab}
