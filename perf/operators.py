"""The operators around a paged cache, as sized cases: attention over whole prompts, attention of new tokens over the
pages, and eviction by accumulated attention weight. One pass is one call of one operator, or for the eviction one step of
a cache at its budget (the new tokens' rows go in, as many tokens are evicted).

A case's keys:
  op        "prompt": causal attention inside packed prompts of different lengths;
            "attend": attention of every sequence's new tokens over its pages, the new tokens' own rows among them;
            "evict": append of new tokens and eviction of the lightest ones down to the budget
  q_heads, kv_heads, head_dim, dtype ("bf16" | "f32")
  batch     sequences
  tokens    prompt: tokens of all prompts together; attend: the longest cache; evict: the budget
  new       attend: most new tokens of a sequence; evict: new tokens of every sequence
  page      tokens per page
  mix       prompt, attend: "even": prompts of equal length, m new tokens everywhere; "ragged": prompts of very different
            lengths, caches of 3/4 to all of `tokens`; "mixed": as ragged, and half of the sequences have one new token,
            the others anything up to `new`
  cut       what the lengths are drawn from
  mass      prompt, attend: the attention weight that every token received is returned, or added to what it has
  fused     prompt: q, k and v are slices of one projection's output
  sinks, recent   evict: the first tokens of a sequence and the newest ones stay whatever they weigh
"""
import math
import random

import torch

own = False

RING = 4  # different steps' inputs that an eviction goes through in turn

# Head counts of the attention layers in use here: grouped-query layers of 7B, 8B and 70B models, ungrouped ones, and one
# with a large group.
HEADS = [(32, 8), (28, 4), (64, 8), (16, 8), (8, 8), (32, 2)]
PAGES = [16, 32, 64, 128]


def _case(name, op, heads, head_dim, dtype, batch, tokens, new=0, page=0, mix="even", cut=0, mass=True, fused=False,
          sinks=0, recent=0):
    c = {} if name is None else {"name": name}
    c.update(op=op, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, dtype=dtype, batch=batch, tokens=tokens,
             new=new, page=page, mix=mix, cut=cut, mass=mass, fused=fused, sinks=sinks, recent=recent)
    return c


def listed():
    return [
        # One short question to an 8B-class model: launches and latency.
        _case("prompt_short", "prompt", (32, 8), 128, "bf16", 1, 129, fused=True),
        # A batch of prompts of a 7B-class model packed one behind another, without eviction in mind.
        _case("prompt_packed", "prompt", (28, 4), 128, "bf16", 7, 12001, mix="ragged", cut=1, mass=False, fused=True),
        # A long document and a shorter one on a 70B-class layer; the weights start the cache's account.
        _case("prompt_long", "prompt", (64, 8), 128, "bf16", 2, 16384, mix="ragged", cut=8),
        # The package's smallest heads in fp32, as a check of a model's numerics runs them.
        _case("prompt_f32", "prompt", (4, 2), 64, "f32", 3, 701, mix="ragged", cut=3),
        # One user's chat, one token: a few megabytes of pages.
        _case("attend_single", "attend", (32, 8), 128, "bf16", 1, 2049, new=1, page=16),
        # A serving batch on a 7B-class layer, ragged caches up to 8k, one token each, weights accounted.
        _case("attend_batch", "attend", (28, 4), 128, "bf16", 64, 8193, new=1, page=32, mix="ragged", cut=4),
        # Few sequences with long caches on a 70B-class layer, no account.
        _case("attend_long", "attend", (64, 8), 128, "bf16", 8, 16385, new=1, page=64, mass=False),
        # A block of a prompt against a 4k cache, weights accounted.
        _case("attend_block", "attend", (32, 8), 128, "bf16", 1, 4224, new=128, page=16),
        # Continuous batching: half of the sequences decode, the others go through blocks of their prompts.
        _case("attend_mixed", "attend", (64, 8), 128, "bf16", 12, 16384, new=512, page=64, mix="mixed", cut=5),
        # A few drafted tokens per sequence to be verified, heads of 64 channels.
        _case("attend_draft", "attend", (32, 8), 64, "bf16", 16, 4099, new=5, page=16, mix="ragged", cut=6, mass=False),
        # The serving batch's eviction: one token in, one token out.
        _case("evict_batch", "evict", (28, 4), 128, "bf16", 64, 8192, new=1, page=32, mix="ragged", cut=4, sinks=4,
              recent=64),
        # Blocks of 512 tokens at a 16k budget on a 70B-class layer.
        _case("evict_block", "evict", (64, 8), 128, "bf16", 8, 16384, new=512, page=64, sinks=4, recent=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the ranges of ``listed``: the three operators in equal shares, sizes over their logarithm."""
    while True:
        op = rng.choice(["prompt", "attend", "evict"])
        heads = rng.choice(HEADS)
        head_dim = 64 if rng.random() < 0.25 else 128
        dtype = "f32" if rng.random() < 0.1 else "bf16"
        cut, mass = rng.randrange(1 << 20), rng.random() < 0.6
        page = rng.choice(PAGES)
        if op == "prompt":
            batch = _log(rng, 1, 12)
            tokens = _log(rng, 1, 1500 if dtype == "f32" else 16384)
            c = _case(None, op, heads, head_dim, dtype, min(batch, tokens), tokens, mix=rng.choice(["even", "ragged"]),
                      cut=cut, mass=mass, fused=rng.random() < 0.5)
        elif op == "attend":
            batch, tokens, new = _log(rng, 1, 64), _log(rng, 16, 16385), 1
            mix = rng.choice(["even", "ragged"])
            if rng.random() < 0.5:
                batch, new = _log(rng, 1, 12), rng.choice([128, _log(rng, 2, 512)])
                mix = rng.choice(["even", "ragged", "mixed"])
            if dtype == "f32":
                batch, tokens, new = min(batch, 4), min(tokens, 2048), min(new, 64)
            c = _case(None, op, heads, head_dim, dtype, batch, tokens, new=min(new, tokens * 3 // 4), page=page, mix=mix,
                      cut=cut, mass=mass)
        else:
            new = rng.choice([1, 1, _log(rng, 2, 512)])
            batch, tokens = _log(rng, 1, 64 if new == 1 else 8), _log(rng, 64, 16384)
            recent = rng.choice([0, tokens // 8])
            c = _case(None, op, heads, head_dim, dtype, batch, tokens, new=min(new, tokens // 4), page=page,
                      mix=rng.choice(["even", "ragged"]), cut=cut, sinks=rng.choice([0, 4]), recent=recent)
        w = work(c)
        if w["bytes"] <= 1.2e9 and w["flops"] <= 2.5e12:
            return c


def _lengths(case):
    """(tokens, new tokens) of every sequence."""
    rng, B, n = random.Random(case["cut"]), case["batch"], case["tokens"]
    if case["op"] == "prompt":
        if case["mix"] == "even":
            lens = [n // B + (1 if b < n % B else 0) for b in range(B)]
        else:
            at = sorted(rng.randint(0, n) for _ in range(B - 1))
            lens = [y - x for x, y in zip([0] + at, at + [n])]
        return lens, list(lens)
    lens = [n if case["mix"] == "even" else rng.randint(max(1, n * 3 // 4), n) for _ in range(B)]
    new = [case["new"]] * B
    if case["mix"] == "mixed":
        new = [1 if rng.random() < 0.5 else rng.randint(1, case["new"]) for _ in range(B)]
    return lens, new


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    """What a model's layer has in hand: the projections of the new tokens, and the sequences' pages.

    Values and keys are normal, with three outlier channels per KV head on the keys and four attention sinks at the start
    of every sequence that the queries lean towards; accumulated weights are positive with a long tail. A sequence's pages
    lie anywhere in the pool, and what its last page has behind its length is whatever was there before.
    """
    dev, d, page = "cuda", case["head_dim"], case["page"]
    B, Hq, Hkv = case["batch"], case["q_heads"], case["kv_heads"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    lens, new = _lengths(case)
    cu, T = _starts(new), sum(new)
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    mult = torch.ones((Hkv, d), device=dev)
    mult[:, torch.randperm(d, generator=g, device=dev)[:3]] = 4.0
    mu = normal(Hkv, d)
    mu = mu / mu.norm(dim=-1, keepdim=True)
    sink, lean = (2.0 * math.sqrt(d)) * mu, 2.0 * mu.repeat_interleave(Hq // Hkv, dim=0)
    state = {"case": case, "lens": lens, "new": new, "starts": cu, "scale": d ** -0.5,
             "cu": torch.tensor(cu, dtype=torch.int32, device=dev)}
    lse = torch.zeros((T, Hq), device=dev)
    if case["op"] == "prompt":
        q, k, v = normal(T, Hq, d) + lean, normal(T, Hkv, d) * mult, normal(T, Hkv, d)
        for b in range(B):
            k[cu[b]:min(cu[b] + 4, cu[b + 1])] = sink
        if case["fused"]:
            qkv = torch.cat([q, k, v], dim=1).to(dtype)
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        else:
            q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
        state.update(q=q, k=k, v=v, o=torch.zeros((T, Hq, d), dtype=dtype, device=dev), lse=lse,
                     mass=torch.zeros((T, Hkv), device=dev) if case["mass"] else None)
        pages = (0, 0, 0)
    else:
        room = [n + (case["new"] if case["op"] == "evict" else 0) for n in lens]  # an eviction begins with an append
        need = [-(-n // page) for n in room]
        n_pages, max_pages = sum(need) + 3, max(need)
        pages = (page, n_pages, max_pages)
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        table = torch.full((B, max_pages), -1, dtype=torch.int32, device=dev)
        at = 0
        for b in range(B):
            table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        K, V = (normal(n_pages, Hkv, page, d) * mult[:, None]).to(dtype), normal(n_pages, Hkv, page, d).to(dtype)
        K[table[:, 0].long(), :, :4] = sink[:, None].to(dtype)
        state.update(K=K, V=V, table=table, len=torch.tensor(lens, dtype=torch.int32, device=dev),
                     mass=normal(n_pages, Hkv, page).exp_() if case["mass"] else None)
    if case["op"] == "attend":
        state.update(q=(normal(T, Hq, d) + lean).to(dtype), o=torch.zeros((T, Hq, d), dtype=dtype, device=dev), lse=lse)
    elif case["op"] == "evict":
        m = case["new"]
        slot = torch.arange(max_pages * page, dtype=torch.int32, device=dev).view(max_pages, 1, page)
        pos = torch.zeros((n_pages, Hkv, page), dtype=torch.int32, device=dev)
        for b in range(B):
            pos[table[b, :need[b]].long()] = slot[:need[b]]
        state.update(pos=pos, seen=state["len"].clone(), budget=state["len"].clone(),
                     out=torch.full((B, Hkv, m), -1, dtype=torch.int32, device=dev),
                     count=torch.zeros((B,), dtype=torch.int32, device=dev), at=0,
                     steps=[{"k": (normal(T, Hkv, d) * mult).to(dtype), "v": normal(T, Hkv, d).to(dtype),
                             "mass": normal(T, Hkv).exp_()} for _ in range(RING)])
    if own:
        import paper_2504_14051_b200 as P

        state["params"] = P.make_paged_params(B, Hq, Hkv, d, *pages, T, max(new), dtype, state["scale"])
        state["workspace"] = P.alloc_paged_workspace(state["params"], dev)
    return state


def _softmax_rows(q, k, v, scale, first):
    """Softmax attention in 32 bits: q [heads, G, rows, d], k and v [heads, n, d]; row i sees the keys up to first + i.
    Returns the output, the log of the sum of exponentials, and the weight that every key received."""
    rows, n = q.shape[2], k.shape[1]
    s = torch.einsum("hgid,hjd->hgij", q, k).mul_(scale)
    hidden = torch.arange(n, device=q.device)[None, :] > first + torch.arange(rows, device=q.device)[:, None]
    s.masked_fill_(hidden, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    p.div_(total)
    return torch.einsum("hgij,hjd->hgid", p, v), (top + total.log()).squeeze(-1), p.sum(dim=(1, 2))


def _attend_sequences(s, keys_of, mass_to):
    """The plain attention of every sequence's rows, a few KV heads at a time so that the logits fit the memory."""
    c = s["case"]
    Hq, Hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    G = Hq // Hkv
    for b, (n, m) in enumerate(zip(s["lens"], s["new"])):
        if m == 0:
            continue
        rows = slice(s["starts"][b], s["starts"][b + 1])
        q = s["q"][rows].float().view(m, Hkv, G, d).permute(1, 2, 0, 3)
        k, v = keys_of(b, n)
        at_once = max(1, min(Hkv, int(2e9) // (G * m * n)))
        for h in range(0, Hkv, at_once):
            heads = slice(h, min(h + at_once, Hkv))
            o, lse, w = _softmax_rows(q[heads], k[heads], v[heads], s["scale"], n - m)
            cols = slice(heads.start * G, heads.stop * G)
            s["o"][rows, cols] = o.permute(2, 0, 1, 3).reshape(m, -1, d).to(s["o"].dtype)
            s["lse"][rows, cols] = lse.permute(2, 0, 1).reshape(m, -1)
            if s["mass"] is not None:
                mass_to(b, n, heads, w)


def _plain_prompt(s):
    def keys_of(b, n):
        rows = slice(s["starts"][b], s["starts"][b + 1])
        return s["k"][rows].float().transpose(0, 1), s["v"][rows].float().transpose(0, 1)

    def mass_to(b, n, heads, w):
        s["mass"][s["starts"][b]:s["starts"][b + 1], heads] = w.t()

    _attend_sequences(s, keys_of, mass_to)


def _plain_attend(s):
    c, page = s["case"], s["case"]["page"]
    Hq, Hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    if max(s["new"]) == 1:  # single tokens: the whole batch at once, padded to the longest cache
        B, G, P = c["batch"], Hq // Hkv, s["table"].shape[1]
        at = s["table"].long().clamp_(min=0)
        k = s["K"][at].permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * page, d).float()
        v = s["V"][at].permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * page, d).float()
        there = (torch.arange(P * page, device=k.device)[None] < s["len"][:, None])[:, None, None]
        x = torch.einsum("bhgd,bhjd->bhgj", s["q"].float().view(B, Hkv, G, d), k).mul_(s["scale"])
        x.masked_fill_(~there, -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        p = (x - top).exp_()
        total = p.sum(dim=-1, keepdim=True)
        p.div_(total)
        s["o"].copy_(torch.einsum("bhgj,bhjd->bhgd", p, v).view(B, Hq, d))
        s["lse"].copy_((top + total.log()).view(B, Hq))
        if s["mass"] is not None:
            used = s["table"] >= 0
            w = p.sum(dim=2).view(B, Hkv, P, page).transpose(1, 2)
            s["mass"].index_add_(0, s["table"][used].long(), w[used])
        return

    def pages_of(b, n):
        return s["table"][b, :-(-n // page)].long()

    def keys_of(b, n):
        at = pages_of(b, n)
        return tuple(x[at].transpose(0, 1).reshape(Hkv, -1, d)[:, :n].float() for x in (s["K"], s["V"]))

    def mass_to(b, n, heads, w):
        at = pages_of(b, n)
        pad = torch.nn.functional.pad(w, (0, at.numel() * page - n)).view(w.shape[0], -1, page).transpose(0, 1)
        s["mass"][at, heads] += pad

    _attend_sequences(s, keys_of, mass_to)


def _plain_evict(s, step):
    c, page, dev = s["case"], s["case"]["page"], s["K"].device
    B, Hkv, m = c["batch"], c["kv_heads"], c["new"]
    d, P = c["head_dim"], s["table"].shape[1]
    at = s["table"].long()
    # append: slot n + i of sequence b lies in page table[b, slot / page]
    n = s["len"].long()
    slot = n[:, None] + torch.arange(m, device=dev)
    to, off = at.gather(1, slot // page).view(-1), (slot % page).view(-1)
    s["K"][to, :, off], s["V"][to, :, off] = step["k"], step["v"]
    s["mass"][to, :, off] = step["mass"]
    s["pos"][to, :, off] = (s["seen"][:, None] + torch.arange(m, dtype=torch.int32, device=dev)).view(-1, 1).expand(-1, Hkv)
    s["seen"] += m
    n = n + m
    # the order of eviction: tokens that have to stay come last, then by weight, then by position
    at0 = at.clamp(min=0)
    w = s["mass"][at0].transpose(1, 2).reshape(B, Hkv, P * page)
    pos = s["pos"][at0].transpose(1, 2).reshape(B, Hkv, P * page)
    stays = (pos < c["sinks"]) | (pos >= (s["seen"] - c["recent"])[:, None, None])
    key = w.view(torch.int32).long().masked_fill_(stays, (1 << 31) - 1) * (1 << 32) + pos.long()
    slots = torch.arange(P * page, device=dev)
    key.masked_fill_(slots >= n[:, None, None], (1 << 63) - 1)
    k = (n - s["budget"].long()).clamp_(min=0)
    most = s["out"].shape[-1]
    light = key.topk(most, dim=-1, largest=False, sorted=True).indices
    light.masked_fill_(torch.arange(most, device=dev) >= k[:, None, None], P * page)
    light = light.sort(dim=-1).values
    taken = light < P * page
    s["out"].copy_(torch.where(taken, light.int(), s["out"]))
    s["count"].copy_(k)
    # the i-th token behind the new length that stays moves into the i-th hole below it
    left = (n - k)[:, None, None]
    gone = torch.zeros((B, Hkv, P * page + 1), dtype=torch.bool, device=dev).scatter_(2, light, True)
    tail = left + torch.arange(most, device=dev)
    moves = (tail < n[:, None, None]) & ~gone.gather(2, tail.clamp(max=P * page).expand(B, Hkv, most))
    rank = (moves.long().cumsum(-1) - 1).clamp_(min=0)
    src = tail.expand(B, Hkv, most).contiguous()
    dst = torch.where(moves, light.gather(2, rank), src)  # (what does not move is written where it is)
    sp, dp = at.gather(1, (src // page).view(B, -1)), at.gather(1, (dst // page).view(B, -1))
    sp, dp = sp.view_as(src), dp.view_as(dst)
    h = torch.arange(Hkv, device=dev)[None, :, None]
    for x in (s["K"], s["V"], s["mass"], s["pos"]):
        x[dp, h, dst % page] = x[sp, h, src % page]
    s["len"].copy_(n - k)


def run(s):
    op = s["case"]["op"]
    if op == "evict":
        step = s["steps"][s["at"] % RING]
        s["at"] += 1
    if own:
        import paper_2504_14051_b200 as P

        p, ws = s["params"], s["workspace"]
        if op == "prompt":
            P.caote_prompt_attend(p, s["q"], s["k"], s["v"], s["cu"], s["o"], s["lse"], s["mass"], ws)
        elif op == "attend":
            P.caote_paged_attend(p, s["q"], s["K"], s["V"], s["mass"], s["table"], s["len"], s["cu"], s["o"], s["lse"], ws)
        else:
            P.caote_paged_append(p, s["K"], s["V"], s["mass"], s["pos"], s["table"], s["len"], s["seen"], step["k"],
                                 step["v"], step["mass"], s["cu"], ws)
            P.caote_paged_evict(p, s["K"], s["V"], s["mass"], s["pos"], s["table"], s["len"], s["seen"], s["budget"],
                                s["case"]["sinks"], s["case"]["recent"], s["out"], s["count"], ws)
    elif op == "prompt":
        _plain_prompt(s)
    elif op == "attend":
        _plain_attend(s)
    else:
        _plain_evict(s, step)
    if op != "evict":
        out = {"o": s["o"], "lse": s["lse"]}
        if s["mass"] is not None:
            out["mass"] = s["mass"]
        return out
    bits = torch.int16 if s["K"].dtype == torch.bfloat16 else torch.int32  # rows are moved, bit for bit
    return {"K": s["K"].view(bits), "V": s["V"].view(bits), "mass": s["mass"], "pos": s["pos"], "len": s["len"],
            "seen": s["seen"], "evicted": s["out"], "count": s["count"]}


def exact(case, seed):
    """Row by row from the definition, in 64 bits."""
    s = prepare(case, seed)
    lens, new, starts, page = s["lens"], s["new"], s["starts"], case["page"]
    Hq, Hkv, dev = case["q_heads"], case["kv_heads"], "cuda"
    G = Hq // Hkv
    if case["op"] == "evict":
        # a token's weight follows its position: what is left of each sequence is its heaviest and its sheltered tokens
        step, m = s["steps"][0], case["new"]
        mass = s["mass"].double().cpu().clone()
        for b, n in enumerate(lens):
            at = s["table"][b].long().cpu()
            for h in range(Hkv):
                w = torch.cat([mass[at[:-(-n // page)], h].reshape(-1)[:n],
                               step["mass"][starts[b]:starts[b + 1], h].double().cpu()])
                held = [j < case["sinks"] or j >= n + m - case["recent"] for j in range(n + m)]
                order = sorted(range(n + m), key=lambda j: (held[j], float(w[j]) if not held[j] else 0.0, j))
                out = set(order[:m])
                fill = [j for j in range(n, n + m) if j not in out]
                kept = w.clone()
                for hole, j in zip(sorted(j for j in out if j < n), fill):
                    kept[hole] = w[j]
                slots = torch.arange(n + m)
                mass[at[slots // page], h, slots % page] = kept
        return {"K": None, "V": None, "mass": mass, "pos": None, "len": None, "seen": None, "evicted": None, "count": None}
    pairs = Hq * sum(m * n for n, m in zip(lens, new))
    if pairs > 2.0e10:
        return None
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device=dev)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=dev)
    mass = None if s["mass"] is None else s["mass"].double()
    if mass is not None and case["op"] == "prompt":
        mass.zero_()
    for b, (n, m) in enumerate(zip(lens, new)):
        for h in range(Hkv if m else 0):
            if case["op"] == "prompt":
                k, v = (s[x][starts[b]:starts[b + 1], h].double() for x in ("k", "v"))
            else:
                slots = torch.arange(n, device=dev)
                where = (s["table"][b].long()[slots // page], h, slots % page)
                k, v = s["K"][where].double(), s["V"][where].double()
            got = torch.zeros(n, dtype=torch.float64, device=dev)
            step = max(1, int(1.0e8) // n)
            for g in range(h * G, (h + 1) * G):
                for i0 in range(0, m, step):
                    i = torch.arange(i0, min(i0 + step, m), device=dev)
                    see = int(n - m + i[-1] + 1)
                    z = (s["q"][starts[b] + i, g].double() @ k[:see].t()) * s["scale"]
                    z = torch.where(torch.arange(see, device=dev)[None] <= (n - m + i)[:, None], z, -math.inf)
                    log = torch.logsumexp(z, dim=1)
                    a = torch.exp(z - log[:, None])
                    o[starts[b] + i, g], lse[starts[b] + i, g] = a @ v[:see], log
                    got[:see] += a.sum(0)
            if mass is not None:
                if case["op"] == "prompt":
                    mass[starts[b]:starts[b + 1], h] = got
                else:
                    mass[where] += got
    out = {"o": o, "lse": lse}
    if mass is not None:
        out["mass"] = mass
    return out


def work(case):
    """Each input read once, each output written once, the two products of attention over the keys that a row sees."""
    Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    e = 2 if case["dtype"] == "bf16" else 4
    lens, new = _lengths(case)
    T = sum(new)
    if case["op"] == "evict":
        # a weight and a position of every token are looked at; rows appended, and as many moved
        n = sum(x + case["new"] for x in lens)
        return {"bytes": float(Hkv * (n * 8 + T * (4 * (2 * d * e) + 28))), "flops": float(Hkv * n)}
    rows = T * (Hq * (2 * d * e + 4))
    if case["op"] == "prompt":
        nbytes = rows + T * Hkv * (2 * d * e + (4 if case["mass"] else 0))
    else:
        nbytes = rows + Hkv * sum(n for n, m in zip(lens, new) if m) * (2 * d * e + (8 if case["mass"] else 0))
    seen = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))
    return {"bytes": float(nbytes), "flops": float(4 * Hq * d * seen)}
