"""Attention over a key-value cache held in pages, the writing of new tokens into it, and its eviction by accumulated
attention weight, as cases that can be prepared, run and measured.

The cache of a layer is a pool of pages [n_pages][n_kv_heads][page_tokens][head_dim] for keys and for values. Row s of the
page table names the pages of sequence s, lens[s] says how many tokens it holds, seen[s] how many it has taken in. Beside the
rows stand, per KV head and token, the attention weight received so far and the token's position.

  append  new tokens of every sequence go to their places behind those that are there
  attend  one or a few query rows of every sequence attend over its tokens (causal among the rows); optionally every token's
          weight becomes decay * weight + the attention it received
  step    append and attend in one call
  evict   append, then every sequence longer than `keep` goes back to `keep` tokens: the first ones and the latest ones stay,
          of the others those of largest weight; kept rows from behind fill the places that became free, in order
"""
import math

import torch

own = False

DEVICE = "cuda:0"

BASE = {
    "op": "attend", "heads_q": 32, "heads_kv": 8, "dim": 128, "dtype": "bf16", "page": 64, "seqs": 1,
    "tokens": 4096,          # tokens of the longest sequence (evict: held between passes)
    "ragged": False,         # lengths spread over a factor of 64, an empty sequence and one of a single token among them
    "rows": 1,               # new tokens (query rows) of every sequence
    "decay": -1.0,           # >= 0: weights are accumulated
    "lse": False,
    "sink": 4, "recent": 0,  # evict
}


def _case(**kw):
    c = dict(BASE)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: one token of one conversation of a thousand tokens
        _case(name="attend-one", tokens=1000, page=16),
        # decoding at the benchmark's batch and context, 16 sequences of 128K tokens
        _case(name="attend-128k", seqs=16, tokens=131072),
        # a served batch of every length, small pages; the log-sum-exp is wanted as well
        _case(name="attend-ragged", heads_q=28, heads_kv=4, seqs=64, tokens=32001, ragged=True, page=16, lse=True),
        # fp32, the small configuration: 4 query heads on one KV head, 64 wide
        _case(name="attend-f32", heads_q=4, heads_kv=1, dim=64, dtype="f32", seqs=2, tokens=4097, page=32, lse=True),
        # the last 16 tokens of a 32K prompt weigh its tokens, before the first eviction
        _case(name="attend-rows", tokens=32768, rows=16, decay=0.0),
        # decoding with weights, so that the cache can be evicted from
        _case(name="step-scored", op="step", seqs=16, tokens=16387, decay=1.0),
        # a large batch of ordinary conversations
        _case(name="step-batch", op="step", seqs=64, tokens=4096, ragged=True, page=16),
        # the write alone: one token of 64 sequences
        _case(name="append-token", op="append", seqs=64, tokens=2048, page=16),
        # the write of a prompt's chunk, four sequences
        _case(name="append-chunk", op="append", seqs=4, tokens=8192, rows=2048),
        # a full cache that gives up one token for each new one
        _case(name="evict-token", op="evict", seqs=16, tokens=5124, recent=1024),
        # a prompt's chunk taken into a bounded cache
        _case(name="evict-chunk", op="evict", tokens=8192, rows=2048, recent=2048),
        # the same with a budget of nearly 128K tokens
        _case(name="evict-long", op="evict", tokens=126976, rows=4096, recent=4096),
    ]



def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend"] * 5 + ["step"] * 3 + ["append"] * 2 + ["evict"] * 4)
    heads_q, heads_kv, dim = rng.choice([(32, 8, 128)] * 4 + [(8, 8, 128), (28, 4, 128), (16, 2, 64), (64, 8, 128), (32, 1, 128), (12, 4, 64)])
    c = dict(op=op, heads_q=heads_q, heads_kv=heads_kv, dim=dim, dtype="f32" if rng.random() < 0.2 else "bf16",
             page=rng.choice([8, 16, 16, 32, 64, 64, 128, 256]))
    if op in ("attend", "step"):
        c["seqs"] = _log_int(rng, 1, 128)
        c["rows"] = rng.choice([1] * 6 + [2, 3, 4, 7, 16])
        c["tokens"] = min(_log_int(rng, 64, 131072), (262144 if c["rows"] > 4 else 1048576) // c["seqs"])
        c["ragged"] = rng.random() < 0.5
        c["decay"] = rng.choice([-1.0, -1.0, 0.0, 0.9, 1.0])
        c["lse"] = rng.random() < 0.4
    elif op == "append":
        c["rows"] = _log_int(rng, 1, 4096)
        c["seqs"] = max(1, min(_log_int(rng, 1, 128), 16384 // c["rows"]))
        c["tokens"] = c["rows"] + _log_int(rng, 1, 4096)
    else:
        c["rows"] = _log_int(rng, 1, 2048)
        c["tokens"] = _log_int(rng, 2 * c["rows"] + 64, 65536)
        c["seqs"] = max(1, min(_log_int(rng, 1, 64), 131072 // c["tokens"]))
        c["recent"] = rng.choice([c["rows"], _log_int(rng, 1, c["tokens"] // 2), c["tokens"] // 2])
    return _case(**c)


def _lens(c):
    """Lengths of the sequences, the new tokens among them; the seed only orders them."""
    n, most = c["seqs"], c["tokens"] + (c["rows"] if c["op"] == "evict" else 0)
    if not c["ragged"]:
        return [most] * n
    lens = [max(c["rows"], int(most * 64.0 ** (-i / max(1, n - 1))) - i % 5) for i in range(n)]
    if n >= 4 and c["op"] != "step":
        lens[-1], lens[-2] = 0, 1                # a padded batch; fewer tokens than query rows where there are several
    return lens


# ------------------------------------------------------------------ inputs

def _normal(shape, gen, dtype):
    out = torch.empty(shape, dtype=dtype, device=DEVICE)
    flat = out.view(-1)
    step = 1 << 28
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n].copy_(torch.randn(n, generator=gen, device=DEVICE))
    return out


def prepare(case, seed):
    c, op = case, case["op"]
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    S, H, P, d, n = c["seqs"], c["heads_kv"], c["page"], c["dim"], c["rows"]
    order = torch.randperm(S, generator=gen, device=DEVICE)
    lens = torch.tensor(_lens(c), dtype=torch.int32, device=DEVICE)[order]
    need = (lens.long() + P - 1) // P
    width = max(1, -(-max(_lens(c)) // P))
    n_pages = sum(-(-x // P) for x in _lens(c)) + 8
    # every sequence's pages are scattered over the pool; places of the table behind a sequence hold no page
    pages = torch.randperm(n_pages, generator=gen, device=DEVICE)
    first = torch.cumsum(need, 0) - need
    place = torch.arange(width, device=DEVICE)
    table = torch.where(place[None] < need[:, None], pages[(first[:, None] + place[None]).clamp(max=n_pages - 1)], -1).int().contiguous()
    # keys: a mean per page and KV head and noise around it, so that attention prefers stretches of text
    k = _normal((n_pages, H, P, d), gen, dtype)
    k.mul_(0.3).add_(torch.randn((n_pages, H, 1, d), generator=gen, device=DEVICE).to(dtype))
    v = _normal((n_pages, H, P, d), gen, dtype)
    st = {"case": c, "op": op, "table": table, "lens": lens, "k": k, "v": v}
    if op in ("attend", "step"):
        st["q"] = _normal((S, n, c["heads_q"], d), gen, dtype)
    if op != "attend":
        st["k_new"] = _normal((S, H, n, d), gen, dtype)
        st["v_new"] = _normal((S, H, n, d), gen, dtype)
    st["seen"] = lens.clone()
    if op == "evict" or c["decay"] >= 0:
        # weights received so far, as sizes a few steps' queries leave
        st["weight"] = torch.exp(torch.randn((n_pages, H, P), generator=gen, device=DEVICE)).mul_(c["heads_q"] / H / c["tokens"])
        st["pos"] = torch.zeros((n_pages, H, P), dtype=torch.int32, device=DEVICE)
    if op == "evict":
        # as earlier evictions leave a cache: the first tokens, the latest ones and some in between, in any order
        held, seen = c["tokens"], 3 * c["tokens"]
        st["lens"].fill_(held)
        st["seen"].fill_(seen)
        some, last = min(c["sink"], held), min(c["recent"], held - min(c["sink"], held))
        mid = held - some - last
        base = torch.cat([torch.arange(some, device=DEVICE), some + 2 * torch.arange(mid, device=DEVICE),
                          torch.arange(seen - last, seen, device=DEVICE)])
        mixed = torch.rand((S, H, held), generator=gen, device=DEVICE).argsort(-1)
        at = _at(st, torch.arange(held, device=DEVICE))
        st["pos"].view(-1)[at.reshape(-1)] = base[mixed].int().reshape(-1)
        st["w_new"] = torch.exp(torch.randn((S, H, n), generator=gen, device=DEVICE)).mul_(c["heads_q"] / H / c["tokens"])
    if own:
        from paper_2412_04757_amd import LtriPagedCache, paged_config
        cfg = paged_config(c["heads_q"], H, d, c["dtype"], page_tokens=P, n_pages=n_pages, table_pages=width, max_seqs=S,
                           rows_max=n if op in ("attend", "step") else 1, weights="weight" in st)
        st["cache"] = LtriPagedCache(cfg, torch.device(DEVICE), k_pages=k, v_pages=v, weight=st.get("weight"), pos=st.get("pos"))
    return st


# ------------------------------------------------------------------ the plain forms

def _at(st, index):
    """Places, in [n_pages][KV head][page_tokens], of the tokens `index` ([L], or [S][1][L]) of every sequence and KV head."""
    c = st["case"]
    P, H = c["page"], c["heads_kv"]
    index = index.expand(c["seqs"], 1, index.shape[-1])
    page = torch.gather(st["table"].long(), 1, (index // P).squeeze(1)).clamp(min=0)
    return (page[:, None] * H + torch.arange(H, device=DEVICE)[:, None]) * P + index % P


def _append(st):
    c = st["case"]
    n = c["rows"]
    index = (st["lens"].long()[:, None] - n + torch.arange(n, device=DEVICE))[:, None]
    at = _at(st, index).reshape(-1)
    st["k"].view(-1, c["dim"])[at] = st["k_new"].reshape(-1, c["dim"])
    st["v"].view(-1, c["dim"])[at] = st["v_new"].reshape(-1, c["dim"])
    if "weight" in st:
        pos = st["seen"][:, None, None] - n + torch.arange(n, dtype=torch.int32, device=DEVICE)
        st["pos"].view(-1)[at] = pos.expand(-1, c["heads_kv"], -1).reshape(-1)
        st["weight"].view(-1)[at] = st["w_new"].reshape(-1) if "w_new" in st else 0.0


def _held(st, pool):
    """A pool's rows as [S][KV head][token][d], in 32 bits."""
    c = st["case"]
    x = pool[st["table"].long().clamp(min=0)].permute(0, 2, 1, 3, 4)
    return x.reshape(c["seqs"], c["heads_kv"], -1, c["dim"]).float()


def _attend(st):
    c = st["case"]
    S, H, n, d = c["seqs"], c["heads_kv"], c["rows"], c["dim"]
    G = c["heads_q"] // H
    lens = st["lens"].long()
    k = _held(st, st["k"])
    key = torch.arange(k.shape[2], device=DEVICE)
    row = torch.arange(n, device=DEVICE).repeat_interleave(G)
    sees = key < (lens[:, None] - (n - 1) + row)[:, None, :, None]                       # [S][1][n G][L]
    q = st["q"].view(S, n, H, G, d).permute(0, 2, 1, 3, 4).reshape(S, H, n * G, d).float()
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).masked_fill_(~sees, -math.inf)
    del k
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    none = total == 0
    v = _held(st, st["v"]).masked_fill_((key >= lens[:, None])[:, None, :, None], 0.0)
    o = (torch.matmul(p, v) / total).masked_fill(none, 0.0)
    out = [o.view(S, H, n, G, d).permute(0, 2, 1, 3, 4).reshape(S, n, c["heads_q"], d).to(st["q"].dtype)]
    if c["lse"]:
        lse = top + total.log()
        out.append(lse.view(S, H, n, G).permute(0, 2, 1, 3).reshape(S, n, c["heads_q"]))
    if c["decay"] >= 0:
        got = p.div_(total).masked_fill_(none, 0.0).sum(2)                               # [S][KV head][L]
        at = _at(st, key)
        there = (key < lens[:, None])[:, None].expand(-1, H, -1)
        w = st["weight"].view(-1)
        w[at[there]] = c["decay"] * w[at[there]] + got[there]
        out.append(st["weight"])
    return out


def _evict(st):
    c = st["case"]
    keep = c["tokens"]
    lens, seen = st["lens"].long()[:, None, None], st["seen"][:, None, None]
    index = torch.arange(st["table"].shape[1] * c["page"], device=DEVICE)
    at = _at(st, index)
    there = index < lens
    pos, w = st["pos"].view(-1)[at], st["weight"].view(-1)[at]
    w = torch.where((pos < c["sink"]) | (pos >= seen - c["recent"]), math.inf, w)
    w = torch.where(there, w, -math.inf)
    rank = torch.empty_like(at)
    rank.scatter_(2, torch.sort(w, dim=2, descending=True, stable=True).indices, index.expand_as(at))
    stays = there & (rank < keep)
    free = at[there & ~stays & (index < keep)]                  # per sequence and KV head as many as ...
    comes = at[stays & (index >= keep)]                         # ... these, both in order
    for pool in (st["k"].view(-1, c["dim"]), st["v"].view(-1, c["dim"]), st["weight"].view(-1), st["pos"].view(-1)):
        pool[free] = pool[comes]
    st["lens"].clamp_(max=keep)


def run(state):
    st = state
    c, op = st["case"], st["op"]
    if op == "evict":
        st["lens"].add_(c["rows"])
        st["seen"].add_(c["rows"])
    if own:
        cache, table, lens = st["cache"], st["table"], st["lens"]
        decay = c["decay"] if c["decay"] >= 0 else None
        lse = torch.empty((c["seqs"], c["rows"], c["heads_q"]), dtype=torch.float32, device=DEVICE) if c["lse"] else None
        if op == "attend":
            got = [cache.attend(table, lens, st["q"], lse=lse, decay=decay)]
        elif op == "step":
            got = [cache.step(table, lens, st["seen"], st["k_new"], st["v_new"], st["q"], lse=lse, decay=decay)]
        else:
            cache.append(table, lens, st["seen"], st["k_new"], st["v_new"], w_new=st.get("w_new"))
            if op == "evict":
                cache.evict(table, lens, st["seen"], c["tokens"], n_sink=c["sink"], n_recent=c["recent"])
            got = []
        if lse is not None:
            got.append(lse)
        if op in ("attend", "step") and decay is not None:
            got.append(st["weight"])
    else:
        if op != "attend":
            _append(st)
        got = _attend(st) if op in ("attend", "step") else []
        if op == "evict":
            _evict(st)
    if op != "attend":
        got += [st["k"], st["v"]]
    if op == "evict":
        got += [st["weight"], st["pos"], st["lens"]]
    elif "pos" in st and op == "step":
        got += [st["pos"]]
    return got


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c, op = case, case["op"]
    elt = 4 if c["dtype"] == "f32" else 2
    H, d, n, S = c["heads_kv"], c["dim"], c["rows"], c["seqs"]
    row = 2 * H * d * elt                                   # a token's key and value rows
    held = sum(_lens(c))
    marks = 8 * H if (op == "evict" or c["decay"] >= 0) else 0     # a token's weights and positions
    new = S * n * (2 * row + marks)                         # read from the call, written to the pages
    table = 4 * sum(-(-x // c["page"]) for x in _lens(c)) + 8 * S
    if op == "append":
        return {"bytes": new + table, "flops": 0}
    if op == "evict":
        # a pass on a cache that was full: the latest tokens stay, of the other new ones as many as of the old ones
        last = min(c["recent"], n)
        moved = S * (last + (n - last) * max(0, c["tokens"] - c["recent"]) // (c["tokens"] + n - c["recent"]))
        return {"bytes": new + 4 * S * n * H + table + held * marks + moved * 2 * (row + marks), "flops": held * H}
    io = 2 * S * n * c["heads_q"] * d * elt + (4 * S * n * c["heads_q"] if c["lse"] else 0)
    seen = 2 * held * 4 * H if c["decay"] > 0 else held * 4 * H if c["decay"] == 0 else 0
    pairs = sum(max(0, x - i) for x in _lens(c) for i in range(n))
    both = S * n * (row + marks) if op == "step" else 0     # a step writes what it has read as keys and values
    return {"bytes": held * row + io + seen + both + table, "flops": 4 * pairs * c["heads_q"] * d}


# ------------------------------------------------------------------ from the definition, in 64 bits

def exact(case, seed):
    """Sequence by sequence and head by head, over rows looked up one sequence at a time."""
    c, op = case, case["op"]
    st = prepare(case, seed)
    P, H, d, n = c["page"], c["heads_kv"], c["dim"], c["rows"]
    G = c["heads_q"] // H
    k, v = st["k"], st["v"]
    if op != "attend":
        k, v = k.double(), v.double()
    weight = st["weight"].double() if "weight" in st else None
    pos = st.get("pos")
    lens = st["lens"].tolist()
    seen = st["seen"].tolist()
    outs, lses = [], []
    for s in range(c["seqs"]):
        T = lens[s] + (n if op == "evict" else 0)
        now = seen[s] + (n if op == "evict" else 0)
        i = torch.arange(T, device=DEVICE)
        pg, sl = st["table"][s].long()[i // P], i % P
        if op != "attend":
            k[pg[T - n:], :, sl[T - n:]] = st["k_new"][s].double().transpose(0, 1)
            v[pg[T - n:], :, sl[T - n:]] = st["v_new"][s].double().transpose(0, 1)
            if weight is not None:
                pos[pg[T - n:], :, sl[T - n:]] = torch.arange(now - n, now, dtype=torch.int32, device=DEVICE)[:, None].expand(-1, H)
                weight[pg[T - n:], :, sl[T - n:]] = st["w_new"][s].double().T if "w_new" in st else 0.0
        if op in ("attend", "step"):
            kk, vv = k[pg, :, sl].double(), v[pg, :, sl].double()           # [T][H][d]
            o = torch.zeros((n, H, G, d), dtype=torch.float64, device=DEVICE)
            l = torch.full((n, H, G), -math.inf, dtype=torch.float64, device=DEVICE)
            got = torch.zeros((H, T), dtype=torch.float64, device=DEVICE)
            for r in range(n):
                seen_keys = T - (n - 1 - r)
                if seen_keys < 1:
                    continue
                for h in range(H):
                    x = st["q"][s, r, h * G:(h + 1) * G].double() @ kk[:seen_keys, h].T / math.sqrt(d)
                    l[r, h] = torch.logsumexp(x, -1)
                    x = torch.exp(x - l[r, h][:, None])
                    o[r, h] = x @ vv[:seen_keys, h]
                    got[h, :seen_keys] += x.sum(0)
            outs.append(o.view(n, c["heads_q"], d))
            lses.append(l.view(n, c["heads_q"]))
            if c["decay"] >= 0:
                weight[pg, :, sl] = c["decay"] * weight[pg, :, sl] + got.T
        if op == "evict" and T > c["tokens"]:
            for h in range(H):
                w, p = weight[pg, h, sl], pos[pg, h, sl]
                fixed = (p < c["sink"]) | (p >= now - c["recent"])
                by_weight = sorted(range(T), key=lambda j, a=fixed.tolist(), b=w.tolist(): (not a[j], 0.0 if a[j] else -b[j], j))
                stays = torch.zeros(T, dtype=torch.bool)
                stays[by_weight[:c["tokens"]]] = True
                free = torch.nonzero(~stays[:c["tokens"]])[:, 0].to(DEVICE)
                comes = torch.nonzero(stays[c["tokens"]:])[:, 0].to(DEVICE) + c["tokens"]
                for pool in (k, v, weight, pos):
                    pool[pg[free], h, sl[free]] = pool[pg[comes], h, sl[comes]]
            lens[s] = c["tokens"]
        elif op == "evict":
            lens[s] = T
    got = []
    if op in ("attend", "step"):
        got.append(torch.stack(outs))
        if c["lse"]:
            got.append(torch.stack(lses))
        if c["decay"] >= 0:
            got.append(weight)
    if op != "attend":
        got += [k, v]
    if op == "evict":
        got += [weight, None, None]
    elif pos is not None and op == "step":
        got += [None]
    return got
