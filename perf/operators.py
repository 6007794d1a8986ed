"""The paged key/value cache on the receiving side of the hand-off, operator by operator: what each call is given, its plain
form in elementary torch operations, the call that a program makes of the package, and what it must move and compute.

Image tokens that a language model has pulled become keys and values of its layers.  Those lie in pages of a few tokens, any
page anywhere in a pool; a request's block table names its pages in order.  Three operators:

  plan    which pages a step's new tokens take and which slot each token gets (`plan_pages`),
  append  the step's keys and values into their slots (`append_pages`),
  attend  the step's queries over the keys and values of their requests (`attend_pages`): causal for the language model's own
          layers, without a mask for layers in which text attends to an image's tokens.
"""
import math
import random

import numpy as np
import torch

own = False  # False: the plain forms; True: the package's operators


def listed():
    return [
        # one request writes one more token: the shortest step there is, all latency
        _plan("plan_one_token", 1, (1, 1), (700, 700), 16, 256),
        # a step of a loaded server: every request writes one token, some of them into a new page, and the batch is padded to a
        # whole number of rows
        _plan("plan_step_500", 500, (1, 1), (0, 8191), 16, 520, padding=12),
        # prefill of many requests at once, from text alone to four tiles of 1601 image tokens and a long prompt
        _plan("plan_prefill_96", 96, (0, 8000), (0, 4100), 64, 200),
        # a small step's keys and values of one layer
        _append("append_step_24", 24, 8, 128, 16, "bf16"),
        # a prefill's, taken out of a fused product's rows
        _append("append_prefill_16001", 16001, 8, 128, 64, "bf16", skipped=37),
        # fp32, a head dim that is no power of two
        _append("append_fp32_2500", 2500, 4, 80, 32, "fp32", skipped=3),
        # one request, one token: the latency between two tokens of a lone user
        _attend("attend_one_token", 32, 8, 128, 16, "bf16", steps=1, step_keys=(1403, 1403)),
        # a step of a loaded server: 64 requests of very different length, one token each
        _attend("attend_step_64", 32, 8, 128, 16, "bf16", steps=64, step_keys=(300, 16000)),
        # one long document, one token, few heads of keys: the keys' axis is all there is to divide
        _attend("attend_long_document", 28, 4, 128, 64, "bf16", steps=1, step_keys=(131071, 131071)),
        # a chunk of a long prompt behind the tokens of an image of four tiles, in one launch with 24 requests' single tokens
        _attend("attend_chunk_and_steps", 32, 8, 128, 16, "bf16", requests=1, new=(2048, 2048), cached=(6404, 6404), steps=24,
                step_keys=(100, 9000)),
        # prefill of four whole prompts with images: the largest product of all
        _attend("attend_prefill_4", 32, 8, 128, 64, "bf16", requests=4, new=(5200, 9000), cached=(0, 0)),
        # text over the tokens of its images in fp32, without a mask: requests with no image have no key at all
        _attend("attend_images_fp32", 16, 16, 64, 32, "fp32", requests=24, new=(1, 90), cached=(0, 5), step_keys=(1, 1), unit=577,
                causal=False),
    ]


def _plan(name, requests, new, cached, page, table, padding=0):
    return {"name": name, "kind": "plan", "requests": requests, "new_low": new[0], "new_high": new[1], "cached_low": cached[0],
            "cached_high": cached[1], "page": page, "table": table, "padding": padding}


def _append(name, rows, kv_heads, dim, page, dtype, skipped=0):
    return {"name": name, "kind": "append", "rows": rows, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype,
            "skipped": skipped}


def _attend(name, heads, kv_heads, dim, page, dtype, requests=0, new=(1, 1), cached=(0, 0), steps=0, step_keys=(1, 1), unit=0,
            causal=True):
    """`requests` with `new` tokens behind `cached` ones and `steps` with one token and `step_keys` keys, that one's among them.
    With a `unit` the keys are a whole number (`cached`) of units, apart from the new tokens."""
    return {"name": name, "kind": "attend", "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype,
            "requests": requests, "new_low": new[0], "new_high": new[1], "cached_low": cached[0], "cached_high": cached[1],
            "steps": steps, "step_low": step_keys[0], "step_high": step_keys[1], "unit": unit, "causal": causal}


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _draw_any(rng):
    kind = rng.choice(("plan", "append", "attend", "attend", "attend"))
    page = rng.choice((8, 16, 32, 64, 128))
    if kind == "plan":
        requests = _log_int(rng, 1, 2000)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, min(8000, 500000 // requests)))
        cached = _log_int(rng, 1, 16000)
        return _plan("", requests, (rng.choice((0, 1)), new), (0, cached), page, (cached + new) // page + rng.randint(1, 9),
                     padding=rng.choice((0, rng.randint(1, 63))))
    heads, kv_heads, dim = rng.choice(((32, 8, 128), (28, 4, 128), (16, 16, 64), (64, 8, 64), (40, 10, 128), (16, 16, 80), (12, 2, 96),
                                       (8, 1, 128), (9, 3, 72), (32, 32, 128)))
    if kind == "append":
        rows = _log_int(rng, 1, 16000)
        return _append("", rows, kv_heads, dim, page, rng.choice(("bf16", "bf16", "fp32")), skipped=rng.randint(0, min(rows - 1, 40)))
    form = rng.choice(("step", "step", "prefill", "mixed", "images"))
    dtype = "bf16" if rng.random() < 0.8 else "fp32"
    steps, keys = _log_int(rng, 1, 128), _log_int(rng, 16, 130000)
    if form == "step":
        return _attend("", heads, kv_heads, dim, page, dtype, steps=steps, step_keys=(max(1, int(keys * rng.random())), keys))
    requests, new = _log_int(rng, 1, 16), _log_int(rng, 2, 9000)
    if form == "images":
        return _attend("", heads, kv_heads, dim, page, dtype, requests=requests, new=(1, min(new, 500)), cached=(0, rng.randint(1, 8)),
                       unit=rng.choice((256, 577, 729, 1601)), causal=False)
    cached = rng.choice((0, _log_int(rng, 1, 16000)))
    return _attend("", heads, kv_heads, dim, page, dtype, requests=requests, new=(max(1, new // 2), new), cached=(cached // 2, cached),
                   steps=steps if form == "mixed" else 0, step_keys=(1, min(keys, 16000)))


def draw(rng):
    most = {"bytes": max(work(c)["bytes"] for c in listed()), "flops": max(work(c)["flops"] for c in listed())}
    while True:
        case = _draw_any(rng)
        w = work(case)
        # an fp32 operation takes nine times as long as a bf16 one
        if w["bytes"] <= most["bytes"] and w["flops"] * (9 if case.get("dtype") == "fp32" else 1) <= most["flops"]:
            del case["name"]
            return case


def _lengths(case):
    """(new tokens, keys) of every request, fixed by the case whatever the seed: the shape of a batch is part of what it costs."""
    numbers = [v for k, v in sorted(case.items()) if isinstance(v, int)]
    rng = random.Random(",".join(map(str, numbers)))
    new = [rng.randint(case["new_low"], case["new_high"]) for _ in range(case["requests"])]
    cached = [rng.randint(case["cached_low"], case["cached_high"]) for _ in range(case["requests"])]
    if case["kind"] == "plan":
        return new, [n + c for n, c in zip(new, cached)]
    keys = [c * case["unit"] if case["unit"] else n + c for n, c in zip(new, cached)]
    steps = [rng.randint(case["step_low"], case["step_high"]) for _ in range(case["steps"])]
    order = list(range(len(new) + len(steps)))
    rng.shuffle(order)
    both = list(zip(new + [1] * len(steps), keys + steps))
    return [both[i][0] for i in order], [both[i][1] for i in order]


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _table(keys, page, width, order):
    """A block table whose requests hold the pages of `order`, one after the other; what lies behind them is left from before."""
    table = order[torch.arange(len(keys) * width, device="cuda") % order.numel()].reshape(len(keys), width).contiguous()
    at = 0
    for r, n in enumerate(keys):
        count = min(-(-n // page), width)
        table[r, :count] = order[at:at + count]
        at += count
    return table


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    page = case["page"]
    state = {"case": case}
    if case["kind"] == "plan":
        new, total = _lengths(case)
        cached = [t - n for n, t in zip(new, total)]
        held = sum(-(-c // page) for c in cached)
        free = sum(-(-t // page) for t in total) - held
        used_before = seed % 7  # the list's entries that earlier steps took
        pages = held + free + used_before + 16
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        state.update(cached=_int32(cached), new=_int32(new), table=_table(cached, page, case["table"], order), pages=pages,
                     free=order[held:].contiguous(), taken=_int32([used_before]), rows=sum(new) + case["padding"])
        return state
    dt, dim, kv_heads = _dtype(case), case["dim"], case["kv_heads"]
    if case["kind"] == "append":
        rows = case["rows"]
        pages = -(-rows // page) + 5
        slots = torch.randperm(pages * page, device="cuda", generator=g)[:rows].sort().values.to(torch.int32)
        if case["skipped"]:  # rows that have no slot
            slots[torch.randperm(rows, device="cuda", generator=g)[:case["skipped"]]] = -1
        heads = 2 * kv_heads  # the queries that lie before the keys in a fused product's rows
        qkv = torch.randn((rows, (heads + 2 * kv_heads), dim), device="cuda", generator=g).to(dt)
        old = torch.randn((2, pages, kv_heads, page, dim), device="cuda", generator=g).to(dt)
        state.update(k=qkv[:, heads:heads + kv_heads], v=qkv[:, heads + kv_heads:], slots=slots, key_pages=old[0], value_pages=old[1])
        return state
    new, keys = _lengths(case)
    need = sum(-(-n // page) for n in keys)
    pages = need + 7
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    width = max(1, max(-(-n // page) for n in keys)) + 2
    rows = sum(new)
    heads = case["heads"]
    # logits of a standard deviation of 2, as far as a trained layer's: some keys matter, most do not
    qkv = torch.randn((rows, heads + 2 * kv_heads, dim), device="cuda", generator=g).mul_(2.0).to(dt)
    state.update(q=qkv[:, :heads], key_pages=torch.empty((pages, kv_heads, page, dim), dtype=dt, device="cuda").normal_(generator=g),
                 value_pages=torch.empty((pages, kv_heads, page, dim), dtype=dt, device="cuda").normal_(generator=g),
                 table=_table(keys, page, width, order), query_offsets=_int32(np.concatenate([[0], np.cumsum(new)])),
                 kv_lens=_int32(keys), new=new, keys=keys, most=max(new))
    return state


def run(state):
    case = state["case"]
    if own:
        import paper_2502_00937_amd as V

        if case["kind"] == "plan":
            plan = V.plan_pages(state["cached"], state["new"], state["table"], state["free"], state["taken"], state["pages"],
                                case["page"], state["rows"])
            return (plan.slots, plan.query_offsets, plan.kv_lens, plan.page_offsets, plan.counts, state["table"])
        if case["kind"] == "append":
            V.append_pages(state["k"], state["v"], state["slots"], state["key_pages"], state["value_pages"])
            return state["key_pages"], state["value_pages"]
        return V.attend_pages(state["q"], state["key_pages"], state["value_pages"], state["table"], state["query_offsets"],
                              state["kv_lens"], state["most"], causal=case["causal"])
    if case["kind"] == "plan":
        return _plain_plan(state, case["page"])
    if case["kind"] == "append":
        return _plain_append(state)
    return _plain_attend(state, case["causal"])


def _plain_plan(s, page):
    """Slots of the step's tokens, in the order of the requests; rows behind the last request's get -1.  A request's tokens fill its
    last page first, then take pages off the free list, which are entered into its row of the block table.  A token whose
    page lies past the row, past the list or outside the pool has no slot."""
    table, free, rows = s["table"], s["free"], s["rows"]
    width, n_free = table.shape[1], free.numel()
    cached, new = s["cached"].long(), s["new"].long()
    ends = new.cumsum(0).clamp(max=rows)
    starts = torch.cat([ends.new_zeros(1), ends])
    asked, new = new.sum(), ends - starts[:-1]
    total = cached + new
    held = ((cached + page - 1) // page).clamp(max=width)
    more = ((total + page - 1) // page).clamp(max=width) - held
    firsts = torch.cat([s["taken"].long(), s["taken"].long() + more.cumsum(0)])
    t = torch.arange(rows, device=table.device)
    inside = t < ends[-1]
    r = torch.searchsorted(ends, t, right=True).clamp(max=cached.numel() - 1)
    at = cached[r] + t - starts[r]
    nth = at // page
    fresh = nth >= held[r]
    index = firsts[r] + nth - held[r]
    number = torch.where(fresh, free[index.clamp(0, n_free - 1)], table[r, nth.clamp(max=width - 1)]).long()
    good = (nth < width) & (number >= 0) & (number < s["pages"]) & ~(fresh & (index >= n_free))
    number = torch.where(good, number, -1)
    slots = torch.where(inside & good, number * page + at % page, -1)
    opens = inside & fresh & (nth < width)
    flat = torch.cat([table.view(-1), table.new_empty(1)])  # the entry behind the table takes what enters none
    flat[torch.where(opens, r * width + nth, table.numel())] = number.to(torch.int32)
    table.copy_(flat[:-1].view_as(table))
    counts = torch.stack([firsts[-1].clamp(max=n_free), asked - (inside & good).sum()])
    return slots.to(torch.int32), starts.to(torch.int32), total.to(torch.int32), firsts.to(torch.int32), counts.to(torch.int32), table


def _plain_append(s):
    """Row i's keys and values of every head to token `slot % page` of page `slot // page`; a slot of -1 is passed over."""
    page = s["key_pages"].shape[2]
    rows = (s["slots"] >= 0).nonzero().view(-1)
    slots = s["slots"][rows].long()
    s["key_pages"][slots // page, :, slots % page] = s["k"][rows]
    s["value_pages"][slots // page, :, slots % page] = s["v"][rows]
    return s["key_pages"], s["value_pages"]


def _plain_attend(s, causal):
    """Request by request and, where its logits are many, some of its queries at a time: softmax(q k^T / sqrt(dim)) v over the keys
    up to the query's own (causal) or all of them; zeros where there is none."""
    q, pages = s["q"], (s["key_pages"], s["value_pages"])
    n, heads, dim = q.shape
    _, kv_heads, page, _ = pages[0].shape
    group = heads // kv_heads
    out = torch.empty((n, heads, dim), dtype=q.dtype, device=q.device)
    first = 0
    for r, (new, keys) in enumerate(zip(s["new"], s["keys"])):
        if new == 0:
            continue
        if keys == 0:
            out[first:first + new] = 0
            first += new
            continue
        held = s["table"][r, :-(-keys // page)].long()
        k, v = (p[held].transpose(0, 1).reshape(kv_heads, -1, dim)[:, :keys].float() for p in pages)
        kt = k.transpose(1, 2).contiguous()
        step = max(1, min(new, (1 << 28) // (heads * keys)))
        for a in range(0, new, step):
            b = min(new, a + step)
            x = q[first + a:first + b].float().view(b - a, kv_heads, group, dim).permute(1, 2, 0, 3).reshape(kv_heads, -1, dim)
            logits = torch.bmm(x, kt) * dim ** -0.5
            if causal:
                last = torch.arange(a, b, device=q.device) + (keys - new)
                hidden = torch.arange(keys, device=q.device)[None, :] > last[:, None]
                logits.view(kv_heads, group, b - a, keys).masked_fill_(hidden, -math.inf)
            top = logits.amax(-1, keepdim=True)
            weights = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
            total = weights.sum(-1, keepdim=True)
            y = torch.bmm(weights, v) / torch.where(total == 0, 1.0, total)
            out[first + a:first + b] = y.view(kv_heads, group, b - a, dim).permute(2, 0, 1, 3).reshape(b - a, heads, dim).to(q.dtype)
        first += new
    return out


def work(case):
    """What a call cannot do without: inputs read once, outputs written once, products over visible keys only."""
    if case["kind"] == "plan":
        new, total = _lengths(case)
        page = case["page"]
        fresh = sum(-(-t // page) - -(-(t - n) // page) for n, t in zip(new, total))
        # lengths in; slots, offsets and key counts out; the free list's pages and the entries they make; the open pages' numbers
        return {"bytes": 4 * (2 * len(new) + sum(new) + case["padding"] + 3 * len(new) + 2 * fresh + len(new)), "flops": 0}
    es = 4 if case["dtype"] == "fp32" else 2
    dim, kv_heads = case["dim"], case["kv_heads"]
    if case["kind"] == "append":
        return {"bytes": 4 * case["rows"] + 2 * 2 * es * (case["rows"] - case["skipped"]) * kv_heads * dim, "flops": 0}
    new, keys = _lengths(case)
    pairs = sum(n * k - (n * (n - 1) // 2 if case["causal"] else 0) for n, k in zip(new, keys))
    table = sum(-(-k // case["page"]) for k in keys)
    return {"bytes": es * dim * (2 * sum(new) * case["heads"] + 2 * sum(k for n, k in zip(new, keys) if n) * kv_heads) + 4 * table,
            "flops": 4 * pairs * case["heads"] * dim}


def exact(case, seed):
    s = prepare(case, seed)
    page = case["page"]
    if case["kind"] == "plan":
        return _exact_plan(s, page)
    if case["kind"] == "append":
        out = [s["key_pages"].double().cpu().numpy(), s["value_pages"].double().cpu().numpy()]
        rows = [s["k"].double().cpu().numpy(), s["v"].double().cpu().numpy()]
        for i, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                for o, x in zip(out, rows):
                    o[slot // page, :, slot % page] = x[i]
        return tuple(torch.from_numpy(o).cuda() for o in out)
    if work(case)["flops"] > 4e12:
        return None
    # head by head in 64 bits, the keys a piece at a time with a running maximum and sum
    q, group, dim = s["q"], case["heads"] // case["kv_heads"], case["dim"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    first = 0
    for r, (new, keys) in enumerate(zip(s["new"], s["keys"])):
        if new and keys:
            at = torch.arange(keys, device="cuda")
            number, place = s["table"][r].long()[at // page], at % page
            for h in range(case["heads"]):
                k, v = (p[number, h // group, place].double() for p in (s["key_pages"], s["value_pages"]))
                x = q[first:first + new, h].double() / math.sqrt(dim)
                m = torch.full((new, 1), -math.inf, dtype=torch.float64, device="cuda")
                z, acc = torch.zeros_like(m), torch.zeros((new, dim), dtype=torch.float64, device="cuda")
                own_key = torch.arange(keys - new, keys, device="cuda").view(-1, 1)
                for a in range(0, keys, 16384):
                    logits = x @ k[a:a + 16384].T.contiguous()
                    if case["causal"]:
                        logits = torch.where(at[a:a + 16384].view(1, -1) <= own_key, logits, -math.inf)
                    up = torch.maximum(m, logits.max(1, keepdim=True).values)
                    safe = torch.where(up.isinf(), 0.0, up)
                    e, shrink = torch.exp(logits - safe), torch.exp(m - safe)
                    z, acc, m = z * shrink + e.sum(1, keepdim=True), acc * shrink + e @ v[a:a + 16384], up
                out[first:first + new, h] = torch.where(z > 0, acc / torch.where(z > 0, z, 1.0), 0.0)
        first += new
    return out


def _exact_plan(s, page):
    table, free = s["table"].cpu().numpy(), s["free"].cpu().numpy()
    slots, starts, total = [], [0], []
    taken = int(s["taken"][0])
    firsts, lost = [taken], 0
    for r, (cached, new) in enumerate(zip(s["cached"].tolist(), s["new"].tolist())):
        fits = min(new, s["rows"] - len(slots))
        lost += new - fits
        for at in range(cached, cached + fits):
            nth = at // page
            if nth < table.shape[1] and at % page == 0:  # this token opens a page
                table[r, nth] = free[taken] if taken < len(free) and 0 <= free[taken] < s["pages"] else -1
                taken += 1
            number = table[r, nth] if nth < table.shape[1] else -1
            slots.append(number * page + at % page if 0 <= number < s["pages"] else -1)
            lost += slots[-1] < 0
        starts.append(starts[-1] + fits)
        total.append(cached + fits)
        firsts.append(taken)
    slots += [-1] * (s["rows"] - len(slots))
    return tuple(torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
                 for x in (slots, starts, total, firsts, [min(taken, len(free)), lost], table))
