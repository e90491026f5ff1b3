"""Timed cases of the operators that keep a coded cache within bounds: window attention, paged attention, masses, eviction.

A case is a dict of plain values:

    path       "window"   cq_window_attn: attention of the newest tokens, a sliding window and the first tokens visible
               "paged"    cq_paged_attn: attention of ragged chunks of new tokens over pages of codes
               "mass"     cq_attn_mass: the attention weight that every cached token receives
               "evict"    cq_evict: the tokens of largest weight move to the front of a smaller cache
    c, b       channels per group and bits per code ("CQ-<c>c<b>b"); head_dim: channels per head
    n_seq, n_q_heads, n_kv_heads
    min_len, max_len   context lengths, spread evenly over [min_len, max_len], dealt out by the seed (new tokens counted)
    capacity   tokens that a sequence's cache has room for
    n_new      query tokens per sequence ("paged": the most; min_new: the least, spread over their logarithm)
    window, sinks   tokens that stay visible behind a query (0: all), and at the front
    page       tokens of a page
    keep, recent    tokens that stay after an eviction, and how many of them are the newest

Vectors follow the library's synthetic recipe: x = A z + mu + 0.1 eps per head, low rank, keys with four outlier channels
(mean +8, std x5); codebooks are draws of that source in fp16, a head's tokens are picks from a few thousand such vectors, coded by their
nearest centroids; queries N(0, 1).  Code buffers have the library's layout [sequence or page][head][block of 16 tokens][group][16].
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
POOL = 2048          # distinct vectors of a head


def _case(name, path, c, n_seq, n_q, n_kv, min_len, max_len, capacity, **more):
    return dict(name=name, path=path, c=c, b=8, head_dim=128, n_seq=n_seq, n_q_heads=n_q, n_kv_heads=n_kv, min_len=min_len,
                max_len=max_len, capacity=capacity, **more)


def listed():
    return [
        # the smallest call: one interactive user with a long conversation, one token, a short window
        _case("window_step_one_user", "window", 8, 1, 32, 8, 20011, 20011, 32768, n_new=1, window=1024, sinks=4),
        # a decode step of a Mistral-7B-shaped layer with its window of 4096, the headline batch
        _case("window_step_gqa", "window", 8, 64, 32, 8, 8192, 16384, 16384, n_new=1, window=4096, sinks=4),
        # a chunk of a long prompt through the same layer
        _case("window_prompt_gqa", "window", 8, 4, 32, 8, 8192, 8192, 8192, n_new=2048, window=4096, sinks=4),
        # a scheduler's odd chunk, every head with keys of its own, 2 bits per channel, a window that ends inside tiles
        _case("window_chunk_4c8b_mha", "window", 4, 3, 32, 32, 1500, 2999, 3001, n_new=333, window=511, sinks=3),
        # a chunk of four prompts over pages of 64 tokens; the largest call
        _case("paged_chunk_gqa", "paged", 8, 4, 32, 8, 8192, 8192, 8192, n_new=2048, min_new=2048, page=64, window=0, sinks=0),
        # a server's mixed batch: prompts in chunks next to conversations that take one token
        _case("paged_mixed_gqa", "paged", 8, 24, 32, 8, 600, 9001, 9216, n_new=512, min_new=1, page=16, window=0, sinks=0),
        # a decode step of the headline batch over pages of 32, ragged contexts
        _case("paged_step_gqa", "paged", 8, 64, 32, 8, 4096, 16384, 16384, n_new=1, min_new=1, page=32, window=0, sinks=0),
        # a decode step of a Llama-2-7B-shaped layer at 2 bits per channel
        _case("paged_step_4c8b_mha", "paged", 4, 16, 32, 32, 4096, 4096, 4096, n_new=1, min_new=1, page=16, window=0, sinks=0),
        # a decode step's weights, added up per cached token
        _case("mass_step_gqa", "mass", 8, 64, 32, 8, 16384, 16384, 16384, n_new=1),
        # the weights that a prompt's last tokens give to the prompt, before it is cut down
        _case("mass_last_queries_gqa", "mass", 8, 4, 32, 8, 5001, 8192, 8192, n_new=32),
        # one user's cache, cut down in between two steps
        _case("evict_one_user", "evict", 8, 1, 32, 8, 4097, 4097, 8192, keep=2048, sinks=4, recent=256),
        # one layer of a Llama-2-13B-shaped batch with long ragged contexts
        _case("evict_mha_ragged", "evict", 8, 32, 40, 40, 8192, 32768, 32768, keep=4096, sinks=4, recent=1024),
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    path = rng.choice(["window", "window", "paged", "paged", "mass", "evict"])
    c = rng.choice([8, 8, 4, 2])
    n_q, n_kv = rng.choice([(32, 8), (32, 32), (40, 40), (8, 1), (12, 4), (1, 1)])
    if path == "evict":
        n_seq = _log(rng, 1, 32)
        last = min(_log(rng, 64, 32768), (32 * 40 * 20480 * 16) // (n_seq * n_kv * (128 // c)))
        first = rng.randint(max(1, last // 4), last)
        keep = _log(rng, 16, max(16, last - 1))
        recent = rng.randint(0, keep // 2)
        case = _case("", path, c, n_seq, n_q, n_kv, first, last, last + rng.randint(0, 64), keep=keep, recent=recent,
                     sinks=rng.randint(0, min(8, keep - recent)))
    else:
        few = rng.random() < 0.5
        n_new = (1 if rng.random() < 0.7 else rng.randint(2, 8)) if few else _log(rng, 9, 64 if path == "mass" else 2048)
        n_seq = _log(rng, 1, 64 if few else 8)
        most = min(16384, (64 * 8 * 16384 * 16) // (n_seq * n_kv * (128 // c)) if few else (4 * 32 * 2048 * 8192) // (n_seq * n_q * n_new))
        last = max(n_new, _log(rng, 64, max(65, most)))
        first = rng.randint(max(n_new, last // 2), last)
        more = dict(n_new=n_new)
        if path != "mass":
            bounded = path == "window" or rng.random() < 0.3
            more.update(window=_log(rng, 16, 4096) if bounded else 0, sinks=rng.randint(0, 70) if bounded else 0)
        if path == "paged":
            more.update(page=rng.choice([16, 32, 48, 64, 128, 256]), min_new=rng.choice([1, n_new]))
        case = _case("", path, c, n_seq, n_q, n_kv, first, last, last + rng.randint(0, 64), **more)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------ inputs

def _host_rng(seed):
    return torch.Generator().manual_seed(seed * 7919 + 11)


def _lengths(case, seed):
    """Context lengths and new tokens of every sequence, on the host."""
    n, g = case["n_seq"], _host_rng(seed)
    lens = torch.linspace(case["min_len"], case["max_len"], n, dtype=torch.float64).round().long()[torch.randperm(n, generator=g)].tolist()
    new = [case.get("n_new", 0)] * n
    if case.get("min_new", case.get("n_new")) != case.get("n_new"):
        spread = torch.linspace(math.log(case["min_new"]), math.log(case["n_new"]), n, dtype=torch.float64).exp().round().long()
        new = spread[torch.randperm(n, generator=g)].tolist()
        new = [min(a, b) for a, b in zip(new, lens)]
    return lens, new


def _vectors(gen, n_heads, n, D, outliers):
    """n vectors of every head (n_heads, n, D) and fp16 centroids from the same source, as draws (n_heads, 256, D)."""
    rank = D // 4
    A = torch.randn(n_heads, rank, D, generator=gen, device=DEV) / rank ** 0.5
    mu = 0.5 * torch.randn(n_heads, 1, D, generator=gen, device=DEV)
    x = torch.randn(n_heads, n + 256, rank, generator=gen, device=DEV) @ A + 0.1 * torch.randn(n_heads, n + 256, D, generator=gen, device=DEV)
    if outliers:
        at = torch.rand(n_heads, 1, D, generator=gen, device=DEV).argsort(-1)[..., :4]
        gain = torch.ones(n_heads, 1, D, device=DEV).scatter_(-1, at, 5.0)
        x = x * gain + torch.zeros(n_heads, 1, D, device=DEV).scatter_(-1, at, 8.0)
    x = (x + mu).half()
    return x[:, :n], x[:, n:]


def _coded(gen, case, slots, keys):
    """Codebooks (n_heads, G, 256, c) fp16 and codes (slots, n_heads, blocks, G, 16) of random picks; slots = (count, blocks)."""
    H, D, c = case["n_kv_heads"], case["head_dim"], case["c"]
    G = D // c
    x, parents = _vectors(gen, H, POOL, D, keys)
    book = parents.view(H, 256, G, c).permute(0, 2, 1, 3).contiguous()
    pool = torch.cdist(x.float().view(H, POOL, G, c).transpose(1, 2).reshape(H * G, POOL, c), book.float().view(H * G, 256, c)).argmin(-1)
    pool = pool.view(H, G, POOL).transpose(1, 2).to(torch.uint8).contiguous()                      # (H, POOL, G)
    count, blocks = slots
    codes = torch.empty(count, H, blocks, G, 16, dtype=torch.uint8, device=DEV)
    for h in range(H):
        pick = torch.randint(0, POOL, (count * blocks, 16), generator=gen, device=DEV)
        codes[:, h] = pool[h][pick].view(count, blocks, 16, G).transpose(2, 3)
    return book, codes


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    lens, new = _lengths(case, seed)
    n, hq, hkv, D, path = case["n_seq"], case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["path"]
    st = dict(case=case, lens=lens, new=new, seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV), scale=D ** -0.5)
    blocks = (case["capacity"] + 15) // 16
    if path == "paged":
        page, per_seq = case["page"], -(-case["capacity"] // case["page"])
        used = [-(-x // page) for x in lens]
        n_pages = sum(used) + 7
        order = torch.randperm(n_pages, generator=_host_rng(seed + 1)).tolist()
        table = torch.full((n, per_seq), -1, dtype=torch.int32)
        at = 0
        for s in range(n):
            table[s, :used[s]] = torch.tensor(order[at:at + used[s]], dtype=torch.int32)
            at += used[s]
        st["page_table"] = table.to(DEV)
        slots = (n_pages, page // 16)
        offs = [0]
        for x in new:
            offs.append(offs[-1] + x)
        st["offsets"] = offs
        st["q_offsets"] = torch.tensor(offs, dtype=torch.int32, device=DEV)
        st["q"] = torch.randn(offs[-1], hq, D, generator=gen, device=DEV).half()
    else:
        slots = (n, blocks)
        if path != "evict":
            st["q"] = torch.randn(n, case["n_new"], hq, D, generator=gen, device=DEV).half()
    st["k_cb"], st["k_codes"] = _coded(gen, case, slots, True)
    if path != "mass":
        st["v_cb"], st["v_codes"] = _coded(gen, case, slots, False)
    if path == "mass":
        # what earlier steps have added up
        st["mass"] = torch.rand(n, hkv, case["capacity"], generator=gen, device=DEV)
        st["mass_out"] = torch.zeros_like(st["mass"])
    if path == "evict":
        # heavy-tailed, and zero (all alike) for tokens that never got any weight
        m = torch.exp(2.0 * torch.randn(n, hkv, case["capacity"], generator=gen, device=DEV) - 3.0)
        st["mass"] = torch.where(torch.rand(m.shape, generator=gen, device=DEV) < 0.1, torch.zeros_like(m), m)
        room = -(-case["keep"] // 16) * 16
        st["room"] = room
        st["k_out"] = torch.zeros(n, hkv, room // 16, D // case["c"], 16, dtype=torch.uint8, device=DEV)
        st["v_out"] = torch.zeros_like(st["k_out"])
        st["mass_out"] = torch.zeros(n, hkv, room, device=DEV)
    if path in ("window", "paged"):
        st["out"] = torch.empty_like(st["q"])
    if own:
        import paper_2405_03917_b200 as cq
        if path == "window":
            size = cq.cq_window_attn_workspace_bytes(n, case["n_new"], hq, hkv, D, case["c"], case["b"], case["capacity"], case["window"], case["sinks"])
        elif path == "paged":
            size = cq.cq_paged_attn_workspace_bytes(n, st["offsets"][-1], case["n_new"], hq, hkv, D, case["c"], case["b"],
                                                    case["page"], st["page_table"].shape[1], case["window"], case["sinks"])
        else:
            size = cq.cq_attn_mass_workspace_bytes(n, max(1, case.get("n_new", 0)), hq, hkv, D, case["c"], case["b"], case["capacity"])
        st["workspace"] = torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------------------------------------------------------ one pass

def run(st):
    if own:
        return _run_own(st)
    path = st["case"]["path"]
    return {"window": _plain_attn, "paged": _plain_attn, "mass": _plain_mass, "evict": _plain_evict}[path](st)


def _run_own(st):
    import paper_2405_03917_b200 as cq
    k = st["case"]
    c, b, cap = k["c"], k["b"], k["capacity"]
    if k["path"] == "window":
        return cq.cq_window_attn(st["q"], st["k_codes"], st["v_codes"], st["k_cb"], st["v_cb"], st["seq_lens"], st["scale"], c, b, cap,
                                 k["window"], k["sinks"], out=st["out"], workspace=st["workspace"])
    if k["path"] == "paged":
        return cq.cq_paged_attn(st["q"], st["q_offsets"], st["k_codes"], st["v_codes"], st["k_cb"], st["v_cb"], st["page_table"], st["seq_lens"],
                                st["scale"], c, b, k["page"], k["n_new"], k["window"], k["sinks"], out=st["out"], workspace=st["workspace"])
    if k["path"] == "mass":
        return cq.cq_attn_mass(st["q"], st["k_codes"], st["k_cb"], st["seq_lens"], st["scale"], c, b, cap, st["mass"],
                               mass_out=st["mass_out"], workspace=st["workspace"])
    kept, lens = cq.cq_evict(st["mass"], st["k_codes"], st["v_codes"], st["seq_lens"], k["head_dim"], c, b, cap, k["keep"], k["sinks"], k["recent"],
                             st["k_out"], st["v_out"], st["mass_out"], st["room"])
    return dict(kept=kept, lens=lens, k=st["k_out"], v=st["v_out"], mass=st["mass_out"])


def _vectors_of(codes, book):
    """codes (heads, blocks, G, 16), book (heads, G, 256, c) -> fp32 vectors (heads, blocks * 16, G * c)."""
    H, nb, G, _ = codes.shape
    c = book.shape[-1]
    at = codes.permute(0, 2, 1, 3).reshape(H, G, nb * 16).long()
    x = torch.gather(book.float(), 2, at.unsqueeze(-1).expand(-1, -1, -1, c))
    return x.permute(0, 2, 1, 3).reshape(H, nb * 16, G * c)


def _blocks_of(st, name, s):
    """The code blocks of sequence s that hold its tokens: (heads, blocks, G, 16)."""
    k, nb = st["case"], -(-st["lens"][s] // 16)
    if k["path"] != "paged":
        return st[name][s, :, :nb]
    pages = st["page_table"][s, :-(-st["lens"][s] // k["page"])].long()
    x = st[name][pages]                                                                          # (pages, heads, blocks of a page, G, 16)
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3], 16)[:, :nb]


def _seen(n, n_new, k):
    """Which of n tokens each of the n_new newest sees: (n_new, n)."""
    t = torch.arange(n, device=DEV)
    pos = torch.arange(n - n_new, n, device=DEV)[:, None]
    seen = t <= pos
    if k.get("window", 0):
        seen &= (t < k["sinks"]) | (t > pos - k["window"])
    return seen


def _plain_weights(st, q, s):
    """Softmax weights of the queries (n_new, heads, D) of sequence s: fp32 (kv heads, heads per kv head, n_new, n)."""
    k, n = st["case"], st["lens"][s]
    H = k["n_kv_heads"]
    keys = _vectors_of(_blocks_of(st, "k_codes", s), st["k_cb"])[:, :n]
    qs = q.float().permute(1, 0, 2).reshape(H, -1, q.shape[0], q.shape[2]) * st["scale"]
    w = torch.matmul(qs, keys.transpose(1, 2).unsqueeze(1))
    w.masked_fill_(~_seen(n, q.shape[0], k), float("-inf"))
    w -= w.amax(-1, keepdim=True)
    w.exp_()
    w /= w.sum(-1, keepdim=True)
    return w


def _plain_attn(st):
    k, out = st["case"], st["out"]
    rows = out.view(-1, k["n_q_heads"], k["head_dim"])
    q = st["q"].view(rows.shape)
    at = 0
    for s in range(k["n_seq"]):
        m = st["new"][s]
        w = _plain_weights(st, q[at:at + m], s)
        values = _vectors_of(_blocks_of(st, "v_codes", s), st["v_cb"])[:, :st["lens"][s]]
        o = torch.matmul(w, values.unsqueeze(1))
        rows[at:at + m] = o.permute(2, 0, 1, 3).reshape(m, k["n_q_heads"], k["head_dim"]).half()
        at += m
    return out


def _plain_mass(st):
    for s in range(st["case"]["n_seq"]):
        n = st["lens"][s]
        w = _plain_weights(st, st["q"][s], s)
        st["mass_out"][s, :, :n] = st["mass"][s, :, :n] + w.sum((1, 2))
    return st["mass_out"]


def _plain_evict(st):
    k = st["case"]
    n, H, cap, keep = k["n_seq"], k["n_kv_heads"], k["capacity"], k["keep"]
    lens = st["seq_lens"].long().view(n, 1, 1)
    t = torch.arange(cap, device=DEV).view(1, 1, cap)
    rank = torch.where((t < k["sinks"]) | (t >= lens - k["recent"]), float("inf"), st["mass"])
    rank = torch.where(t < lens, rank, float("-inf"))
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    left = lens.clamp(max=keep)
    j = torch.arange(order.shape[-1], device=DEV).view(1, 1, -1)
    kept = torch.where(j < left, order, cap).sort(-1).values                                      # ascending, the missing ones last
    here = kept < cap
    at = kept.clamp(max=cap - 1)
    res = dict(kept=torch.full((n, H, keep), -1, dtype=torch.int32, device=DEV))
    res["kept"][..., :kept.shape[-1]] = torch.where(here, kept, -1).int()
    res["lens"] = left.view(n).int()
    for name in ("k", "v"):
        rm = st[name + "_codes"].transpose(3, 4).reshape(n, H, -1, st["k_codes"].shape[3])       # (n, H, tokens, G)
        x = torch.zeros(n, H, st["room"], rm.shape[-1], dtype=torch.uint8, device=DEV)
        x[:, :, :at.shape[-1]] = torch.where(here.unsqueeze(-1), torch.gather(rm, 2, at.unsqueeze(-1).expand(-1, -1, -1, rm.shape[-1])), 0)
        res[name] = x.view(n, H, -1, 16, rm.shape[-1]).transpose(3, 4).contiguous()
    st["mass_out"][..., :at.shape[-1]] = torch.where(here, torch.gather(st["mass"], 2, at), st["mass_out"][..., :at.shape[-1]])
    res["mass"] = st["mass_out"]
    return res


# ------------------------------------------------------------------------------------------ what a pass cannot do without

def _pairs(n, m, window, sinks):
    """(query, visible token) pairs of m queries at the end of n tokens, and the tokens that any of them sees."""
    if not window:
        return sum(range(n - m + 1, n + 1)), n
    pairs = 0
    for p in range(n - m, n):
        first = max(0, p - window + 1)
        pairs += p + 1 - first + min(first, sinks)
    first = max(0, n - m - window + 1)
    return pairs, n - first + min(first, sinks)


def work(case):
    lens, new = _lengths(case, 1)
    H, hq, D, c = case["n_kv_heads"], case["n_q_heads"], case["head_dim"], case["c"]
    G = D // c
    if case["path"] == "evict":
        kept = sum(min(x, case["keep"]) for x in lens)
        return {"bytes": H * (4 * sum(lens) + kept * (2 * (2 * G + 4) + 4)), "flops": 2 * H * sum(lens)}
    tensors = 1 if case["path"] == "mass" else 2
    data = sum(new) * hq * D * 2 * tensors
    flops = seen = 0
    for n, m in zip(lens, new):
        pairs, tokens = _pairs(n, m, case.get("window", 0), case.get("sinks", 0))
        data += H * tokens * (G * tensors + (8 if tensors == 1 else 0)) + 4
        if case["path"] == "paged":
            data += 4 * -(-n // case["page"])
        flops += 2 * tensors * D * hq * pairs
        seen += tokens
    data += tensors * H * D * 2 * min(256, seen)                        # the centroids that so many codes can name
    return {"bytes": data, "flops": flops}


# ------------------------------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["path"] == "evict":
        return dict(kept=None, lens=None, k=None, v=None, mass=_exact_evicted(st, case))
    H, hq, D, G, c = case["n_kv_heads"], case["n_q_heads"], case["head_dim"], case["head_dim"] // case["c"], case["c"]
    R = hq // H
    res = st["mass"].new_zeros(st["mass"].shape, dtype=torch.float64) if case["path"] == "mass" else st["q"].new_zeros(st["q"].shape, dtype=torch.float64)
    flat = res.view(-1, hq, D) if case["path"] != "mass" else None
    q = st["q"].reshape(-1, hq, D)
    group = torch.arange(G, device=DEV)
    row = 0
    for s in range(case["n_seq"]):
        n, m = st["lens"][s], st["new"][s]
        t = torch.arange(n, device=DEV)
        if case["path"] == "paged":
            where = st["page_table"][s].long()[t // case["page"]]
            block, slot = (t % case["page"]) // 16, t % 16
        else:
            where, block, slot = torch.full_like(t, s), t // 16, t % 16
        pos = n - m + torch.arange(m, device=DEV)
        hidden = t[None, :] > pos[:, None]
        if case.get("window", 0):
            hidden |= (t[None, :] <= pos[:, None] - case["window"]) & (t[None, :] >= case["sinks"])
        for h in range(H):
            def rebuilt(codes, book):
                j = codes[where[:, None], h, block[:, None], group[None, :], slot[:, None]].long()
                return book[h].double()[group[None, :], j].reshape(n, D)
            keys = rebuilt(st["k_codes"], st["k_cb"])
            values = rebuilt(st["v_codes"], st["v_cb"]) if case["path"] != "mass" else None
            for r in range(h * R, h * R + R):
                p = torch.softmax((q[row:row + m, r].double() @ keys.T * st["scale"]).masked_fill(hidden, float("-inf")), -1)
                if values is None:
                    res[s, h, :n] += p.sum(0)
                else:
                    flat[row:row + m, r] = p @ values
            if values is None:
                res[s, h, :n] += st["mass"][s, h, :n].double()
        row += m
    return res


def _exact_evicted(st, case):
    """The masses that stay, moved without a rounding: the order of (not forced, -mass, index) as one whole number per token."""
    res = torch.zeros(st["mass_out"].shape, dtype=torch.float64, device=DEV)
    for s, n in enumerate(st["lens"]):
        t = torch.arange(n, device=DEV)
        m = st["mass"][s, :, :n].contiguous()
        number = (m.view(torch.int32).long() << 20) + ((1 << 20) - 1 - t)                         # masses are not negative: their bits are in order
        number[:, :case["sinks"]] = 1 << 60
        number[:, max(0, n - case["recent"]):] = 1 << 60
        least = number.topk(min(n, case["keep"]), dim=-1).values[:, -1:]
        stays = number >= least
        for h in range(case["n_kv_heads"]):
            left = m[h][stays[h]].double()
            res[s, h, :left.shape[0]] = left
    return res
