"""What the operators of token-generating experts are measured on, each call by itself.

A transformer-shaped expert that answers with tokens keeps the keys and values of its requests in a cache of fixed-size blocks.
Once per step it plans (which blocks every request owns, where every new token's row goes); in every layer it appends the new
tokens' keys and values and attends to what is cached; at the end it draws each request's next token from the logits.  A case
is one of those calls: "plan", "append", "attend" or "sample".

Requests differ in length as they do in a running service: lengths are spread evenly between the case's bounds by the case's
own `mix` number, so that the work of a case is known without its inputs; blocks are scattered over the pool, as in a pool that
has been allocated and freed for a while, and rows that no request has written hold what an earlier request left there.
"""
import math
import random

import numpy as np
import torch

own = False


def listed():
    return [
        # every request of a running batch grows by one token: the step that repeats thousands of times
        dict(name="plan_step_192", kind="plan", requests=192, block=16, lo=1, hi=4000, new_lo=1, new_hi=1, single=1.0, done=0.0, pool=60000, mix=1),
        # a busy service: chunks of prompts beside single tokens, finished requests that give their blocks back
        dict(name="plan_mixed_1500", kind="plan", requests=1500, block=32, lo=0, hi=6000, new_lo=0, new_hi=300, single=0.6, done=0.06, pool=300001, mix=2),
        # one layer's keys and values of a batch of single tokens
        dict(name="append_48", kind="append", tokens=48, pad=0, kv=8, dim=128, block=16, pool=1500, layout="token"),
        # one layer's keys and values of prompt chunks, a few rows of padding at the end of a fixed-size step
        dict(name="append_8000", kind="append", tokens=8000, pad=37, kv=8, dim=128, block=16, pool=1500, layout="head"),
        # one token of one request of the repository's transformer shape (12 heads of 64): the latency of an idle service
        dict(name="attend_1_of_613", kind="attend", requests=1, heads=12, kv=12, dim=64, block=16, lo=612, hi=612, new_lo=1, new_hi=1, single=1.0,
             window=0, layout="token", mix=3),
        # an ordinary batch of single tokens, four query heads to a head of the cache, lengths all over
        dict(name="attend_96_tokens", kind="attend", requests=96, heads=32, kv=8, dim=128, block=16, lo=50, hi=5000, new_lo=1, new_hi=1, single=1.0,
             window=0, layout="token", mix=4),
        # few requests with very long histories, eight query heads to a head of the cache
        dict(name="attend_3_long", kind="attend", requests=3, heads=32, kv=4, dim=128, block=64, lo=90000, hi=131071, new_lo=1, new_hi=1, single=1.0,
             window=0, layout="head", mix=5),
        # chunks of prompts and single tokens in one step, a head width that is no power of two
        dict(name="attend_40_mixed", kind="attend", requests=40, heads=24, kv=8, dim=96, block=32, lo=0, hi=3000, new_lo=64, new_hi=700, single=0.7,
             window=0, layout="token", mix=6),
        # two long prompts, the largest matrix products
        dict(name="attend_2_prompts", kind="attend", requests=2, heads=32, kv=8, dim=128, block=16, lo=0, hi=2000, new_lo=7001, new_hi=9001, single=0.0,
             window=0, layout="token", mix=7),
        # the next token of one request
        dict(name="sample_1", kind="sample", rows=1, vocab=50001, dtype="f32", greedy=0.0, top_k=40, top_p=0.95, min_p=0.0, plain=0.0, spread=3.0),
        # a batch whose requests each bring their own settings, some greedy, some without any filter
        dict(name="sample_96", kind="sample", rows=96, vocab=128000, dtype="f32", greedy=0.15, top_k=100, top_p=0.9, min_p=0.02, plain=0.1, spread=3.0),
        # many requests, logits as a bf16 product leaves them, a nucleus only
        dict(name="sample_600", kind="sample", rows=600, vocab=32003, dtype="bf16", greedy=0.0, top_k=0, top_p=0.92, min_p=0.0, plain=0.0, spread=2.5),
    ]


def _spread(rng, lo, hi):
    """An integer whose logarithm is uniform over the range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "sample", "sample"])
    mix = rng.randrange(1, 1 << 30)
    if kind == "plan":
        requests = _spread(rng, 1, 1500)
        block = rng.choice([8, 16, 32, 64])
        hi = _spread(rng, 16, 6000)
        return dict(kind=kind, requests=requests, block=block, lo=0, hi=hi, new_lo=rng.choice([0, 1]), new_hi=_spread(rng, 1, min(300, 150000 // requests)),
                    single=rng.choice([0.0, 0.5, 1.0]), done=rng.choice([0.0, 0.05]), pool=requests * (hi // block + 2) + requests * (300 // block + 2), mix=mix)
    if kind == "append":
        tokens = _spread(rng, 1, 8000)
        kv, dim = rng.choice([1, 2, 4, 8, 12]), rng.choice([64, 80, 96, 128])
        if kv * dim > 1024:
            kv = 8
        return dict(kind=kind, tokens=tokens, pad=rng.choice([0, 0, 5]), kv=kv, dim=dim, block=rng.choice([8, 16, 64]), pool=1500,
                    layout=rng.choice(["token", "head"]))
    if kind == "sample":
        rows = _spread(rng, 1, 300)
        return dict(kind=kind, rows=rows, vocab=_spread(rng, 1000, min(160000, 12000000 // rows)), dtype=rng.choice(["f32", "bf16"]),
                    greedy=rng.choice([0.0, 0.2]), top_k=rng.choice([0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 0.95, 0.8, 0.5]),
                    min_p=rng.choice([0.0, 0.0, 0.05]), plain=rng.choice([0.0, 0.2]), spread=rng.choice([1.5, 3.0, 5.0]))
    kv, group = rng.choice([(12, 1), (8, 4), (4, 8), (8, 3), (2, 7), (1, 16), (5, 5)])
    case = dict(kind=kind, requests=1, heads=kv * group, kv=kv, dim=rng.choice([64, 64, 80, 96, 128, 128]), block=rng.choice([8, 16, 32, 64, 128]))
    form = rng.choice(["tokens", "tokens", "mixed", "prompt"])
    if form == "tokens":
        requests = _spread(rng, 1, 200)
        hi = _spread(rng, 64, min(131000, 250000 // requests))
        case.update(requests=requests, lo=rng.choice([0, hi // 2, hi]), hi=hi, new_lo=1, new_hi=rng.choice([1, 1, 3]), single=rng.choice([0.5, 1.0]))
    elif form == "mixed":
        case.update(requests=rng.randint(2, 40), lo=0, hi=_spread(rng, 64, 4000), new_lo=rng.choice([0, 10]), new_hi=_spread(rng, 12, 700),
                    single=rng.choice([0.3, 0.7]))
    else:
        new = _spread(rng, 100, 6000)
        case.update(requests=rng.randint(1, 2), lo=0, hi=rng.choice([0, 1000, 4000]), new_lo=new, new_hi=new + rng.randint(0, 99), single=0.0)
    case.update(window=rng.choice([0, 0, 0, _spread(rng, 32, 2048)]), layout=rng.choice(["token", "head"]), mix=mix)
    return case


# ---- lengths ---------------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens in the cache and tokens to come of every request; -1 tokens to come: the request is finished."""
    rng = random.Random(case["mix"])
    n = case["requests"]
    have = [case["lo"] + (case["hi"] - case["lo"]) * (i + 1) // n for i in range(n)]
    rng.shuffle(have)
    new = [1 if rng.random() < case["single"] else rng.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    if sum(new) == 0:
        new[0] = 1
    for i in range(n):
        if rng.random() < case.get("done", 0.0):
            new[i] = -1
    return have, new


def _blocks(tokens, block):
    return (tokens + block - 1) // block


def _visible(case):
    """Pairs (query token, cached token) that the attention of a case looks at, and cached tokens that some query sees."""
    pairs = rows = 0
    for h, m in zip(*_lengths(case)):
        w = case["window"]
        if m == 0:
            continue
        if w == 0:
            pairs += m * h + m * (m + 1) // 2
            rows += h + m
        else:
            short = max(0, min(m, w - h))                     # queries that still see everything before them
            pairs += short * h + short * (short + 1) // 2 + (m - short) * w
            rows += min(h + m, w + m - 1)
    return pairs, rows


# ---- inputs ----------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _randn(gen, *shape):
    """bf16 normal values; large tensors in pieces, so that the 32-bit values they come from stay small."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    for s in range(0, flat.numel(), 1 << 27):
        piece = flat[s:s + (1 << 27)]
        piece.copy_(torch.randn(piece.shape, generator=gen, device="cuda"))
    return out


def _cache(case, pool, gen):
    """Key and value caches, as views [block][token][head][channel] of the case's layout."""
    if case["layout"] == "token":
        return [_randn(gen, pool, case["block"], case["kv"], case["dim"]) for _ in range(2)]
    return [_randn(gen, pool, case["kv"], case["block"], case["dim"]).permute(0, 2, 1, 3) for _ in range(2)]


def _prepare_plan(case, seed):
    rng = np.random.default_rng(seed)
    block, pool = case["block"], case["pool"]
    have, new = _lengths(case)
    n, width = len(have), max(_blocks(h + max(m, 0), block) for h, m in zip(have, new)) + 1
    order = rng.permutation(pool).astype(np.int32)
    table = np.full((n, width), -1, np.int32)
    at = 0
    for r, h in enumerate(have):
        b = _blocks(h, block)
        table[r, :b] = order[at:at + b]
        at += b
    head, count = int(rng.integers(pool)), pool - at
    ring = np.full(pool, -1, np.int32)
    ring[(head + np.arange(count)) % pool] = order[at:]
    cap = sum(max(m, 0) for m in new) + 5
    empty = dict(dtype=torch.int32, device="cuda")
    return dict(have=_ints(have), add=_ints(new), table=torch.from_numpy(table).cuda(), ring=torch.from_numpy(ring).cuda(), state=_ints([head, count]), cap=cap,
                width=width, seq_len=torch.empty(n, **empty), q_off=torch.empty(n + 1, **empty), slot=torch.empty(cap, **empty),
                position=torch.empty(cap, **empty), next=torch.empty(4, **empty))


def _prepare_append(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    k_cache, v_cache = _cache(case, case["pool"], gen)
    n, pad = case["tokens"], case["pad"]
    # one product gives queries, keys and values of a token side by side; the new rows are slices of it
    qkv = _randn(gen, n + pad, 3 * case["kv"], case["dim"])
    slot = torch.full((n + pad,), -1, dtype=torch.int32, device="cuda")
    slot[:n] = torch.randperm(case["pool"] * case["block"], generator=gen, device="cuda")[:n].int()
    kept = torch.arange(n, device="cuda")
    return dict(k=qkv[:, case["kv"]:2 * case["kv"]], v=qkv[:, 2 * case["kv"]:], slot=slot, k_cache=k_cache, v_cache=v_cache, kept=kept)


def _prepare_attend(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    have, new = _lengths(case)
    block, kv, dim, heads = case["block"], case["kv"], case["dim"], case["heads"]
    total = [h + m for h, m in zip(have, new)]
    owned = [_blocks(t, block) for t in total]
    pool, width = sum(owned) + 7, max(owned) + 1
    order = np.random.default_rng(seed).permutation(pool).astype(np.int32)
    table = np.full((len(have), width), -1, np.int32)
    at = 0
    for r, b in enumerate(owned):
        table[r, :b] = order[at:at + b]
        at += b
    off = [0]
    for m in new:
        off.append(off[-1] + m)
    k_cache, v_cache = _cache(case, pool, gen)
    qkv = _randn(gen, off[-1], heads + 2 * kv, dim)
    state = dict(q=qkv[:, :heads], k_cache=k_cache, v_cache=v_cache, table=torch.from_numpy(table).cuda(), seq_len=_ints(total), q_off=_ints(off),
                 off=off, total=total, most=max(new), scale=1.0 / math.sqrt(dim), out=torch.empty(off[-1], heads, dim, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty(off[-1], heads, dtype=torch.float32, device="cuda"))
    if own:
        from paper_2503_02354_amd import binding as B
        need = B.coe_kv_attention_workspace(len(have), off[-1], max(new), heads, kv, dim)
        state["work"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    return state


def _prepare_sample(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    n, v = case["rows"], case["vocab"]
    # a language model's logits: a broad bulk and a tail of likely tokens
    logits = case["spread"] * torch.randn(n, v, generator=gen, device="cuda")
    if case["dtype"] == "bf16":
        logits = logits.bfloat16()
    noise = torch.empty(n, v, device="cuda").exponential_(generator=gen)
    plain = rng.random(n) < case["plain"]
    temperature = np.where(rng.random(n) < case["greedy"], 0.0, rng.choice([0.6, 0.8, 1.0, 1.2], n)).astype(np.float32)
    top_k = np.where(plain, 0, case["top_k"]).astype(np.int32)
    top_p = np.where(plain, 1.0, case["top_p"]).astype(np.float32)
    min_p = np.where(plain, 0.0, case["min_p"]).astype(np.float32)
    state = dict(logits=logits, noise=noise, token=torch.empty(n, dtype=torch.int32, device="cuda"), logprob=torch.empty(n, device="cuda"))
    for name, value in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p)):
        state[name] = torch.from_numpy(value).cuda()
    if own:
        from paper_2503_02354_amd import binding as B
        state["work"] = torch.empty(max(B.coe_sample_workspace(n, v), 1), dtype=torch.uint8, device="cuda")
    return state


def prepare(case, seed):
    state = {"plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend, "sample": _prepare_sample}[case["kind"]](case, seed)
    state["case"] = case
    return state


# ---- the calls -------------------------------------------------------------------------------------------------
def _own_run(state):
    from paper_2503_02354_amd import binding as B
    case, stream = state["case"], torch.cuda.current_stream().cuda_stream
    s = {name: t.data_ptr() for name, t in state.items() if isinstance(t, torch.Tensor)}
    kind = case["kind"]
    if kind == "plan":
        B.coe_kv_plan(case["requests"], case["block"], case["pool"], state["width"], state["cap"], s["have"], s["add"], s["ring"], s["state"], s["table"],
                      s["seq_len"], s["q_off"], s["slot"], s["position"], s["next"], stream)
        return _outputs(state)
    if kind == "sample":
        B.coe_sample_tokens(case["rows"], case["vocab"], B.COE_DT_F32 if case["dtype"] == "f32" else B.COE_DT_BF16, s["logits"], state["logits"].stride(0),
                            s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["noise"], state["noise"].stride(0), s["token"], s["logprob"],
                            s["work"], state["work"].numel(), stream)
        return _outputs(state)
    kc = state["k_cache"]
    cache = B.coe_kv_cache(B.COE_DT_BF16, kc.shape[0], case["block"], case["kv"], case["dim"], s["k_cache"], s["v_cache"], *kc.stride()[:3])
    if kind == "append":
        B.coe_kv_append(cache, state["slot"].numel(), s["k"], *state["k"].stride()[:2], s["v"], *state["v"].stride()[:2], s["slot"], stream)
    else:
        B.coe_kv_attention(cache, case["requests"], state["off"][-1], state["most"], case["heads"], case["window"], state["scale"],
                           s["q"], *state["q"].stride()[:2], s["q_off"], s["seq_len"], s["table"], state["table"].shape[1],
                           s["out"], *state["out"].stride()[:2], s["lse"], s["work"], state["work"].numel(), stream)
    return _outputs(state)


def _outputs(state):
    names = {"plan": ("seq_len", "q_off", "slot", "position", "next", "table", "ring"), "append": ("k_cache", "v_cache"), "attend": ("out", "lse"),
             "sample": ("token", "logprob")}[state["case"]["kind"]]
    return {name: state[name] for name in names}


def _plain_plan(state):
    case, block, pool, cap = state["case"], state["case"]["block"], state["case"]["pool"], state["cap"]
    have, add, table, ring = state["have"].long(), state["add"].long(), state["table"], state["ring"]
    head, count = state["state"][0].long(), state["state"][1].long()
    n, width = table.shape
    device = table.device
    grow = add >= 0
    new = torch.where(grow, add, torch.zeros_like(add))
    old_blocks = torch.div(have + block - 1, block, rounding_mode="floor")
    need = torch.where(grow, torch.div(have + new + block - 1, block, rounding_mode="floor") - old_blocks, torch.zeros_like(have))
    # first come, first served: from the first request that does not fit on, none grows
    fits = (torch.cumsum(need, 0) <= count) & (torch.cumsum(new, 0) <= cap) & (have + new <= width * block)
    given = torch.cumprod((fits | ~grow).long(), 0)
    need, new = need * given, new * given
    need_off, freed = torch.cumsum(need, 0) - need, torch.where(grow, torch.zeros_like(have), old_blocks)
    freed_off = torch.cumsum(freed, 0) - freed
    column = torch.arange(width, device=device)[None, :]
    # blocks of finished requests go to the ring's end, new ones come from its front
    back = column < freed[:, None]
    to = torch.where(back, (head + count + freed_off[:, None] + column) % pool, torch.full_like(back, pool, dtype=torch.long))
    wider = torch.cat([ring, ring[:1]])                       # what no finished request gives back lands behind the end
    wider[to] = table
    ring.copy_(wider[:pool])
    fresh = (column >= old_blocks[:, None]) & (column < (old_blocks + need)[:, None])
    table.copy_(torch.where(fresh, ring[(head + need_off[:, None] + column - old_blocks[:, None]) % pool], table))
    state["seq_len"].copy_(torch.where(grow, have + new, torch.zeros_like(have)))
    ends = torch.cumsum(new, 0)
    state["q_off"][0] = 0
    state["q_off"][1:] = ends
    token = torch.arange(cap, device=device)
    marks = torch.zeros(cap + 1, dtype=torch.long, device=device).index_add_(0, torch.clamp(ends, max=cap), torch.ones_like(ends))
    owner = torch.clamp(torch.cumsum(marks, 0)[:cap], max=n - 1)
    position = have[owner] + token - (ends - new)[owner]
    used = token < ends[-1]
    position = torch.where(used, position, torch.full_like(position, -1))
    page = torch.clamp(torch.div(position, block, rounding_mode="floor"), min=0, max=width - 1)
    slot = table[owner, page].long() * block + position % block
    state["slot"].copy_(torch.where(used, slot, torch.full_like(slot, -1)))
    state["position"].copy_(position)
    state["next"].copy_(torch.stack([(head + need.sum()) % pool, count - need.sum() + freed.sum(), given.sum(), ends[-1]]))


def _plain_append(state):
    block = state["case"]["block"]
    kept = state["kept"]
    slot = state["slot"][kept].long()
    page, row = torch.div(slot, block, rounding_mode="floor"), slot % block
    state["k_cache"][page, row] = state["k"][kept]
    state["v_cache"][page, row] = state["v"][kept]


def _plain_attend(state):
    case = state["case"]
    kv, dim, heads, window = case["kv"], case["dim"], case["heads"], case["window"]
    group = heads // kv
    for r, (total, begin, end) in enumerate(zip(state["total"], state["off"], state["off"][1:])):
        m = end - begin
        if m == 0:
            continue
        pages = state["table"][r, :_blocks(total, case["block"])].long()
        k = state["k_cache"][pages].reshape(-1, kv, dim)[:total].float().permute(1, 2, 0).contiguous()            # [kv][dim][total]
        v = state["v_cache"][pages].reshape(-1, kv, dim)[:total].float().permute(1, 0, 2).contiguous()            # [kv][total][dim]
        key = torch.arange(total, device=k.device)
        for s in range(0, m, 1024):
            c = min(1024, m - s)
            q = state["q"][begin + s:begin + s + c].float().reshape(c, kv, group, dim).permute(1, 0, 2, 3).reshape(kv, c * group, dim)
            at = (total - m + s + torch.arange(c, device=k.device)).repeat_interleave(group)[:, None]
            seen = key[None, :] <= at
            if window:
                seen = seen & (key[None, :] > at - window)
            score = torch.matmul(q, k) * state["scale"]
            score = score.masked_fill_(~seen, -math.inf)
            top = score.amax(-1, keepdim=True)
            p = torch.exp(score.sub_(top))
            norm = p.sum(-1, keepdim=True)
            o = torch.matmul(p, v) / norm
            state["out"][begin + s:begin + s + c] = o.reshape(kv, c, group, dim).permute(1, 0, 2, 3).reshape(c, heads, dim).bfloat16()
            state["lse"][begin + s:begin + s + c] = (top + torch.log(norm)).reshape(kv, c, group).permute(1, 0, 2).reshape(c, heads)


def _plain_sample(state):
    rows = state["logits"].shape[0]
    for s in range(0, rows, 64):
        part = slice(s, min(rows, s + 64))
        x = state["logits"][part].float()
        temperature = state["temperature"][part, None]
        greedy = temperature == 0
        z = x / torch.where(greedy, torch.ones_like(temperature), temperature)
        z = z - z.amax(-1, keepdim=True)
        log_sum = torch.log(torch.exp(z).sum(-1, keepdim=True))
        # descending logits, equal ones by index: the filters keep a prefix of this order
        value, index = torch.sort(z, dim=-1, descending=True, stable=True)
        rank = torch.arange(x.shape[1], device=x.device)[None, :]
        k = state["top_k"][part, None]
        keep = (k <= 0) | (rank < k)
        p = torch.where(keep, torch.exp(value), torch.zeros_like(value))
        before = torch.cumsum(p, -1) - p
        top_p = state["top_p"][part, None]
        keep = keep & ((top_p >= 1) | (before < top_p * p.sum(-1, keepdim=True))) & (torch.exp(value) >= state["min_p"][part, None])
        race = value - torch.log(state["noise"][part].gather(1, index))
        race = torch.where(keep, race, torch.full_like(race, -math.inf))
        race = torch.where(greedy, torch.where(rank == 0, torch.zeros_like(race), torch.full_like(race, -math.inf)), race)
        best = race.amax(-1, keepdim=True)
        token = torch.where(race == best, index, torch.full_like(index, x.shape[1])).amin(-1, keepdim=True)
        state["token"][part] = token[:, 0].int()
        state["logprob"][part] = (z.gather(1, token) - log_sum)[:, 0]


def run(state):
    if own:
        return _own_run(state)
    {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[state["case"]["kind"]](state)
    return _outputs(state)


# ---- work and exact results ------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "plan":
        have, new = _lengths(case)
        tokens, n = sum(max(m, 0) for m in new), len(new)
        grown = sum(_blocks(h + m, case["block"]) - _blocks(h, case["block"]) for h, m in zip(have, new) if m >= 0)
        freed = sum(_blocks(h, case["block"]) for h, m in zip(have, new) if m < 0)
        # lengths in and out, offsets, slots and positions; every block that changes hands is read once and written once
        return {"bytes": 4 * (2 * n + 2 * n + 1 + 2 * (tokens + 5) + 6 + 2 * (grown + freed)), "flops": 0}
    if kind == "append":
        return {"bytes": 2 * 2 * 2 * case["tokens"] * case["kv"] * case["dim"] + 4 * (case["tokens"] + case["pad"]), "flops": 0}
    if kind == "attend":
        pairs, rows = _visible(case)
        tokens = sum(_lengths(case)[1])
        return {"bytes": 2 * 2 * rows * case["kv"] * case["dim"] + 2 * 2 * tokens * case["heads"] * case["dim"] + 4 * tokens * case["heads"],
                "flops": 4 * pairs * case["heads"] * case["dim"]}
    n, v = case["rows"], case["vocab"]
    # the logits; the random numbers of the tokens that no filter takes away: all of a row's where it has none
    free = case["plain"] if case["top_k"] or case["top_p"] < 1 or case["min_p"] > 0 else 1.0
    return {"bytes": int(n * v * (4 if case["dtype"] == "f32" else 2) + 4 * n * v * free * (1 - case["greedy"]) + n * 24), "flops": 4 * n * v}


def _exact_plan(case, seed):
    st = _prepare_plan(case, seed)
    block, pool, width, cap = case["block"], case["pool"], st["width"], st["cap"]
    have, add = st["have"].tolist(), st["add"].tolist()
    table, ring = st["table"].cpu().numpy(), st["ring"].cpu().numpy()
    head, count = st["state"].tolist()
    seq_len, q_off, slot, position = [], [0], [], []
    taken = returned = served = 0
    closed = False
    for r, (h, m) in enumerate(zip(have, add)):
        before = -(-h // block)
        if m < 0:
            for j in range(before):
                ring[(head + count + returned) % pool] = table[r, j]
                returned += 1
            seq_len.append(0)
            served += not closed
        else:
            more = -(-(h + m) // block) - before
            closed = closed or taken + more > count or q_off[-1] + m > cap or h + m > width * block
            if closed:
                m = 0
            else:
                served += 1
                for j in range(more):
                    table[r, before + j] = ring[(head + taken) % pool]
                    taken += 1
            seq_len.append(h + m)
            for i in range(h, h + m):
                position.append(i)
                slot.append(int(table[r, i // block]) * block + i % block)
        q_off.append(len(slot))
    tokens = len(slot)
    slot += [-1] * (cap - tokens)
    position += [-1] * (cap - tokens)
    out = dict(seq_len=seq_len, q_off=q_off, slot=slot, position=position, next=[(head + taken) % pool, count - taken + returned, served, tokens])
    out = {name: torch.tensor(value, dtype=torch.int32, device="cuda") for name, value in out.items()}
    out["table"], out["ring"] = torch.from_numpy(table).cuda(), torch.from_numpy(ring).cuda()
    return out


def _exact_append(case, seed):
    st = _prepare_append(case, seed)
    k, v = st["k_cache"].double(), st["v_cache"].double()
    slots = st["slot"].tolist()
    new_k, new_v = st["k"].double(), st["v"].double()
    for t, s in enumerate(slots):
        if s >= 0:
            k[s // case["block"], s % case["block"]] = new_k[t]
            v[s // case["block"], s % case["block"]] = new_v[t]
    return dict(k_cache=k, v_cache=v)


def _exact_attend(case, seed):
    st = _prepare_attend(case, seed)
    have, new = _lengths(case)
    kv, block, window = case["kv"], case["block"], case["window"]
    group = case["heads"] // kv
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    begin = 0
    for r, (h, m) in enumerate(zip(have, new)):
        slots = torch.arange(h + m, device="cuda")
        page, row = st["table"][r][slots // block].long(), slots % block
        for g in range(kv if m else 0):
            k, v = st["k_cache"][page, row, g].double(), st["v_cache"][page, row, g].double()
            for a in range(g * group, (g + 1) * group):
                for s in range(0, m, 2048):
                    e = min(m, s + 2048)
                    last = h + e                                       # keys that the last query of the piece sees
                    q = st["q"][begin + s:begin + e, a].double()
                    x = (q @ k[:last].t().contiguous()) * st["scale"]
                    i = torch.arange(h + s, h + e, device="cuda")[:, None]
                    j = slots[None, :last]
                    x[(j > i) | ((i - j >= window) if window else (j < 0))] = -math.inf
                    total = torch.logsumexp(x, 1)
                    out[begin + s:begin + e, a] = torch.exp(x - total[:, None]) @ v[:last]
                    lse[begin + s:begin + e, a] = total
        begin += m
    return dict(out=out, lse=lse)


def _exact_sample(case, seed):
    st = _prepare_sample(case, seed)
    token, logprob = [], []
    settings = [st[name].double().cpu().numpy() for name in ("temperature", "top_k", "top_p", "min_p")]
    for r in range(case["rows"]):
        temperature, top_k, top_p, min_p = (s[r] for s in settings)
        x = st["logits"][r].double().cpu().numpy()
        z = x / (temperature if temperature > 0 else 1.0)
        w = np.exp(z - z.max())
        if temperature == 0:
            pick = int(np.argmax(x))
        else:
            # everything that could be kept, most likely first
            n = int(top_k) if 0 < top_k < len(x) else len(x)
            likely = np.flatnonzero(x >= np.partition(x, len(x) - n)[len(x) - n])
            order = likely[np.argsort(-x[likely], kind="stable")][:n]
            mass = np.cumsum(w[order])
            cut = len(order)
            if top_p < 1:
                cut = int(np.searchsorted(mass, top_p * mass[-1], side="left")) + 1
            order = order[:cut]
            order = order[(w[order] >= min_p)]
            noise = st["noise"][r].cpu().numpy().astype(np.float64)[order]
            with np.errstate(divide="ignore"):
                score = z[order] - np.log(noise)
            pick = int(order[score == score.max()].min())
        token.append(pick)
        logprob.append(float(z[pick] - z.max() - np.log(w.sum())))
    return dict(token=torch.tensor(token, dtype=torch.int32, device="cuda"), logprob=torch.tensor(logprob, dtype=torch.float64, device="cuda"))


def exact(case, seed):
    return {"plan": _exact_plan, "append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["kind"]](case, seed)
