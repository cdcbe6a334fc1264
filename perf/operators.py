"""The attention block that stands between the qkv and the output projection of a decoder layer, as timed cases.

A pass calls one of three operators of a serving program that keeps its keys and values in pages:

* ``assign``: requests bring new tokens; pages are taken from the stack of free ones, block tables get them, and every token
  gets its position and its slot in the cache (``dmr_kv_assign``);
* ``append``: the output of the qkv projection becomes queries, and keys and values in the cache: a norm for each query and key
  head, the rotation by position, and the write into the pages (``dmr_kv_append``);
* ``attend``: each new token attends to its request's keys in the pages up to itself (``dmr_attn_paged``).

A cache is two pools of pages, [page][kv head][block of 16 tokens][16 x head_dim]; within a block the elements lie in pieces of 16
bytes, ``pc`` elements each (8 bf16 or 16 e4m3): keys [head_dim / pc][16 tokens][pc], values [16 / pc][head_dim][pc tokens].
"""
import math
import random

import torch

own = False

EPS = 1e-6
THETA = 1e6                     # base of the rotation's frequencies
K_SCALE, V_SCALE = 0.0625, 0.03125   # what one step of an e4m3 cache stands for
MAX_KV_BYTES = 7.5e8            # of the keys and values that one drawn pass reads
MAX_FLOPS = 1.0e12
MAX_SCORES = 2.0e9              # padded scores of the plain form


def _assign(name, requests, new, old, page):
    """`new` tokens for a request at most, spread evenly from one on; `old` likewise."""
    return {"name": name, "kind": "assign", "requests": requests, "new": new, "old": old, "page": page}


def _append(name, rows, heads, kv_heads, dim, page, cache, norm=True, interleaved=False):
    return {"name": name, "kind": "append", "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "cache": cache, "norm": norm, "interleaved": interleaved}


def _attend(name, requests, new, kv_min, kv_max, heads, kv_heads, dim, page, cache):
    """`new` tokens for each request, the last of kv_min .. kv_max keys, spread evenly."""
    return {"name": name, "kind": "attend", "requests": requests, "new": new, "kv_min": kv_min, "kv_max": kv_max, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "cache": cache}


def listed():
    return [
        # one decode step of a batch of rollouts: one token each, few requests need a page
        _assign("assign_64req_decode", 64, 1, 9000, 16),
        # an admission of ragged prompts
        _assign("assign_200req_prompts", 200, 160, 700, 64),
        # one decode row of the 7B-class decoder: what a step pays for each layer besides the weights
        _append("append_1row_bf16", 1, 32, 8, 128, 64, "bf16"),
        # a batch of rollouts, keys and values kept in 8 bits, no norms, adjacent pairs rotated
        _append("append_67rows_e4m3_d64", 67, 24, 8, 64, 32, "e4m3", False, True),
        # a prefill chunk
        _append("append_8192rows_bf16", 8192, 32, 8, 128, 64, "bf16"),
        # one agent, an early step: a short history
        _attend("decode_1req_1003keys_bf16", 1, 1, 1003, 1003, 32, 8, 128, 64, "bf16"),
        # sixteen concurrent environments, histories of different lengths
        _attend("decode_16req_to_9000_bf16", 16, 1, 300, 9000, 32, 8, 128, 64, "bf16"),
        # a large batch on an 8-bit cache
        _attend("decode_96req_to_8100_e4m3", 96, 1, 1, 8100, 32, 8, 128, 32, "e4m3"),
        # one very long history
        _attend("decode_1req_131071keys_bf16", 1, 1, 131071, 131071, 32, 8, 128, 128, "bf16"),
        # a few tokens at once, as when drafted ones are verified, with two query heads to a key head and small pages
        _attend("verify_12req_5new_d64_e4m3", 12, 5, 900, 4700, 16, 8, 64, 16, "e4m3"),
        # a chunk of a long prompt over what is in the cache
        _attend("chunk_2048_of_32768_bf16", 1, 2048, 32768, 32768, 32, 8, 128, 64, "bf16"),
        # ragged prompts prefilled together into an 8-bit cache
        _attend("prefill_7req_1500_e4m3", 7, 1500, 1500, 2300, 32, 8, 128, 64, "e4m3"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


def draw(rng):
    kind = rng.choice(("assign",) + ("append",) * 3 + ("attend",) * 6)
    page = rng.choice((16, 32, 64, 128, 256))
    if kind == "assign":
        requests = _log_int(rng, 1, 512)
        return {k: v for k, v in _assign("", requests, _log_int(rng, 1, max(1, 32768 // requests)), _log_int(rng, 1, 20000), page).items()
                if k != "name"}
    kv_heads = rng.choice((1, 2, 3, 4, 8, 8, 16))
    heads = kv_heads * rng.choice((1, 2, 3, 4, 4, 5, 7, 8))
    dim = rng.choice((64, 128, 128))
    cache = rng.choice(("bf16", "bf16", "e4m3"))
    if kind == "append":
        rows = min(_log_int(rng, 1, 8192), 50331648 // ((heads + 2 * kv_heads) * dim))
        c = _append("", rows, heads, kv_heads, dim, page, cache, rng.random() < 0.7, rng.random() < 0.25)
    else:
        size = {"bf16": 2, "e4m3": 1}[cache]
        requests = _log_int(rng, 1, 128)
        per_key = 2 * kv_heads * dim * size
        kv_max = max(1, min(_log_int(rng, 1, 131072), int(MAX_KV_BYTES / (requests * per_key))))
        new = 1 if rng.random() < 0.5 else min(kv_max, _log_int(rng, 1, 4096))
        new = max(1, min(new, int(MAX_FLOPS / (4.0 * heads * dim * requests * kv_max)),
                         int(MAX_SCORES / (float(requests) * heads * kv_max))))
        kv_min = min(kv_max, max(new, _log_int(rng, 1, kv_max)))
        c = _attend("", requests, new, kv_min, kv_max, heads, kv_heads, dim, page, cache)
    return {k: v for k, v in c.items() if k != "name"}


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly: what a case's requests bring, in the order before they are shuffled."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lens(case, seed):
    """New tokens and keys before them, for each request in its order."""
    n = case["requests"]
    if case["kind"] == "assign":
        new, old = _spread(1, case["new"], n), _spread(0, case["old"], n)
    else:
        keys = _spread(case["kv_min"], case["kv_max"], n)
        new, old = [min(case["new"], k) for k in keys], [k - min(case["new"], k) for k in keys]
    rng = random.Random(seed)
    if case["kind"] == "assign":
        rng.shuffle(new)
        rng.shuffle(old)
        return new, old
    both = list(zip(new, old))
    rng.shuffle(both)
    return [a for a, _ in both], [b for _, b in both]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _pool_shapes(case, pages):
    pc = 8 if case["cache"] == "bf16" else 16
    head = (pages, case["kv_heads"], case["page"] // 16)
    return head + (case["dim"] // pc, 16, pc), head + (16 // pc, case["dim"], pc)


def _cached(values, case):
    return values.to(torch.bfloat16 if case["cache"] == "bf16" else torch.float8_e4m3fn)


def _scales(case):
    return (1.0, 1.0) if case["cache"] == "bf16" else (K_SCALE, V_SCALE)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    st = dict(case)
    P = case["page"]
    if case["kind"] == "append":
        T, H, Hk, D = case["rows"], case["heads"], case["kv_heads"], case["dim"]
        st["qkv"] = normal(T, (H + 2 * Hk) * D).mul_(1.5).to(torch.bfloat16)
        st["gamma_q"] = (1.0 + 0.2 * normal(D)).to(torch.bfloat16) if case["norm"] else None
        st["gamma_k"] = (1.0 + 0.2 * normal(D)).to(torch.bfloat16) if case["norm"] else None
        st["inv_freq"] = (THETA ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)).float()
        # consecutive tokens of a few requests, far into their histories, in pages from all over the pool
        runs = max(1, T // 300) if T > 64 else T
        length = -(-T // runs)
        pages_each = length // P + 2
        first = torch.randint(0, 100000, (runs,), generator=gen, device="cuda")
        table = torch.randperm(runs * pages_each, generator=gen, device="cuda").view(runs, pages_each)
        t = torch.arange(T, device="cuda")
        pos = first[t // length] + t % length
        at = first[t // length] % P + t % length
        st["positions"] = pos.int()
        st["slots"] = (table[t // length, at // P] * P + at % P).int()
        k_shape, v_shape = _pool_shapes(case, runs * pages_each)
        st["k"] = torch.zeros(k_shape, dtype=torch.uint8, device="cuda").to(torch.bfloat16 if case["cache"] == "bf16" else torch.float8_e4m3fn)
        st["v"] = torch.zeros(v_shape, dtype=torch.uint8, device="cuda").to(st["k"].dtype)
        st["q"] = torch.empty((T, H * D), dtype=torch.bfloat16, device="cuda")
        if own:
            st["pool"] = _pool(st)
        return st
    new, old = _lens(case, seed)
    n = len(new)
    if case["kind"] == "assign":
        width = (case["old"] + case["new"]) // P + 2
        held = [-(-o // P) for o in old]
        need = [-(-(a + o) // P) - h for a, o, h in zip(new, old, held)]
        pages = sum(held) + sum(need) + 64
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        col = torch.arange(width, device="cuda")[None, :]
        start = torch.cumsum(_ints([0] + held[:-1]), 0)[:, None]
        h = _ints(held)[:, None]
        st["table"] = torch.where(col < h, order[(start + col).clamp(max=pages - 1)], torch.full((), -1, dtype=torch.int32, device="cuda"))
        st["free_pages"] = order[sum(held):].contiguous()
        st["free_count"] = _ints([pages - sum(held)])
        st["new_tokens"], st["lens"], st["rows"] = _ints(new), _ints(old), sum(new)
        # what a step keeps of its requests: where their rows begin, their lengths, positions, slots, pages left and refusals
        st["step"] = tuple(torch.empty(m, dtype=torch.int32, device="cuda") for m in (n + 1, n, sum(new), sum(new), 2))
        return st
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    lens = [a + o for a, o in zip(new, old)]
    width = -(-max(lens) // P) + 1
    held = [-(-k // P) for k in lens]
    pages = sum(held) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    col = torch.arange(width, device="cuda")[None, :]
    start = torch.cumsum(_ints([0] + held[:-1]), 0)[:, None]
    st["kv_lens"] = _ints(lens)
    st["query_start"] = _ints([sum(new[:i]) for i in range(n + 1)])
    # entries behind a request's last page are never filled in
    st["table"] = torch.where(col < _ints(held)[:, None], order[(start + col).clamp(max=pages - 1)],
                              torch.full((), -1, dtype=torch.int32, device="cuda"))
    # slots that no token was written to hold what the memory held before: here NaN
    k_scale, v_scale = _scales(case)
    k_shape, v_shape = _pool_shapes(case, pages)
    tok = torch.arange(width * P, device="cuda")[None, :]
    slot = (st["table"].long().repeat_interleave(P, 1) * P + tok % P)[tok < st["kv_lens"][:, None]]
    blank = torch.ones(pages * P, dtype=torch.bool, device="cuda")
    blank[slot] = False
    blank = blank.view(pages, 1, P // 16, 16)
    pc = k_shape[-1]
    st["k"] = _cached(normal(*k_shape).div_(k_scale).masked_fill_(blank[:, :, :, None, :, None], math.nan), case)
    st["v"] = _cached(normal(*v_shape).div_(v_scale).masked_fill_(blank.view(pages, 1, P // 16, 16 // pc, 1, pc), math.nan), case)
    # scores of deviation 2: some rows have a few keys that matter, most spread
    st["q"] = normal(sum(new), H * D).mul_(2.0).to(torch.bfloat16)
    st["out"] = torch.empty_like(st["q"])
    if own:
        import paper_2602_02711_amd as dmr
        st["pool"] = _pool(st)
        need = dmr.dmr_attn_paged_workspace_bytes(sum(new), n, H, Hk, D, max(new))
        st["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return st


def _pool(st):
    """The program's handle of its cache."""
    import paper_2602_02711_amd as dmr
    k_scale, v_scale = _scales(st)
    return dmr.KvCache(st["k"], st["v"], k_scale, v_scale)


def run(st):
    if own:
        import paper_2602_02711_amd as dmr
        if st["kind"] == "assign":
            step = dmr.dmr_kv_assign(st["new_tokens"], st["lens"], st["free_pages"], st["free_count"], st["table"], st["page"], st["rows"],
                                     out=st["step"])
            return tuple(step) + (st["table"],)
        if st["kind"] == "append":
            dmr.dmr_kv_append(st["pool"], st["qkv"], st["heads"], st["positions"], st["slots"], gamma_q=st["gamma_q"], gamma_k=st["gamma_k"],
                              eps=EPS, inv_freq=st["inv_freq"], interleaved=st["interleaved"], out=st["q"])
            return st["q"], st["k"], st["v"]
        return dmr.dmr_attn_paged(st["pool"], st["q"], st["heads"], st["query_start"], st["kv_lens"], st["table"], st["new"], _softmax_scale(st),
                                  out=st["out"], workspace=st["workspace"])
    return {"assign": _plain_assign, "append": _plain_append, "attend": _plain_attend}[st["kind"]](st)


def _softmax_scale(st):
    return st["dim"] ** -0.5


def _plain_assign(st):
    P, T, table = st["page"], st["rows"], st["table"]
    new = st["new_tokens"].clamp(min=0).long()
    old = torch.where(st["lens"] < 0, -1 - st["lens"], st["lens"]).long()
    free = st["free_count"].long()
    end = torch.cumsum(new, 0)
    first, last = (old + P - 1) // P, (old + new + P - 1) // P
    fits = (last <= table.shape[1]) & (end <= T)
    need = torch.where(fits, last - first, torch.zeros_like(first))
    upto = torch.cumsum(need, 0)
    good = fits & ((need == 0) | (upto <= free))
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    nth = (upto - need)[:, None] + col - first[:, None]
    fresh = good[:, None] & (col >= first[:, None]) & (col < last[:, None])
    page = st["free_pages"][(free - 1 - nth).clamp(0, st["free_pages"].numel() - 1)]
    table.copy_(torch.where(fresh, page, table))
    start = torch.cat([torch.zeros_like(end[:1]), end]).clamp(max=T)
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=new.numel() - 1)
    live = good[b] & (t < start[-1])
    pos = torch.where(live, old[b] + t - start[b], torch.zeros_like(t))
    slot = table[b, (pos // P).clamp(max=table.shape[1] - 1)].long() * P + pos % P
    left = torch.stack([free[0] - torch.where(good, need, torch.zeros_like(need)).sum(), (~good).sum()])
    return (start.int(), torch.where(good, old + new, -1 - old).int(), pos.int(), torch.where(live, slot, torch.full_like(slot, -1)).int(),
            left.int(), table)


def _plain_append(st):
    T, H, Hk, D, P = st["rows"], st["heads"], st["kv_heads"], st["dim"], st["page"]
    x = st["qkv"].float().view(T, H + 2 * Hk, D)
    q, k, v = x[:, :H], x[:, H:H + Hk], x[:, H + Hk:]
    if st["gamma_q"] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * st["gamma_q"].float()
    if st["gamma_k"] is not None:
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * st["gamma_k"].float()
    # angles of far positions in 64 bits
    angle = st["positions"].double()[:, None, None] * st["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def rotate(y):
        if st["interleaved"]:
            a, b = y[..., 0::2], y[..., 1::2]
            return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    k_scale, v_scale = _scales(st)
    st["q"].copy_(rotate(q).reshape(T, H * D))
    pc = st["k"].shape[-1]
    keep = (st["slots"] >= 0).nonzero()[:, 0]
    slot = st["slots"][keep].long()
    page, block, tok = slot // P, slot % P // 16, slot % 16
    raw = torch.int16 if st["cache"] == "bf16" else torch.uint8
    k8 = _cached((rotate(k)[keep] / k_scale).clamp(-448, 448) if st["cache"] != "bf16" else rotate(k)[keep], st)
    v8 = _cached((v[keep] / v_scale).clamp(-448, 448) if st["cache"] != "bf16" else v[keep], st)
    st["k"].view(raw)[page, :, block, :, tok, :] = k8.view(raw).view(-1, Hk, D // pc, pc)
    st["v"].view(raw)[page, :, block, tok // pc, :, tok % pc] = v8.view(raw).view(-1, Hk, D)
    return st["q"], st["k"], st["v"]


def _gathered(st):
    """Keys and values of each request in their order, [request][kv head][key][dim], in 32 bits."""
    Hk, D = st["kv_heads"], st["dim"]
    n, width = st["table"].shape
    at = st["table"].clamp(min=0).long()
    raw = torch.int16 if st["cache"] == "bf16" else torch.uint8
    k_scale, v_scale = _scales(st)
    k = st["k"].view(raw)[at].view(st["k"].dtype).float().mul_(k_scale)
    v = st["v"].view(raw)[at].view(st["v"].dtype).float().mul_(v_scale)
    # [n][width][Hk][blocks] and then keys [D / pc][16][pc], values [16 / pc][D][pc]
    k = k.permute(0, 2, 1, 3, 5, 4, 6).reshape(n, Hk, width * st["page"], D)
    v = v.permute(0, 2, 1, 3, 4, 6, 5).reshape(n, Hk, width * st["page"], D)
    return k, v


def _plain_attend(st):
    H, Hk, D, most = st["heads"], st["kv_heads"], st["dim"], st["new"]
    G, n = H // Hk, st["table"].shape[0]
    start, lens = st["query_start"].long(), st["kv_lens"].long()
    count = start[1:] - start[:-1]
    T = st["q"].shape[0]
    k, v = _gathered(st)
    key = torch.arange(k.shape[2], device="cuda")
    v = torch.where((key[None, :] < lens[:, None])[:, None, :, None], v, torch.zeros((), device="cuda"))
    i = torch.arange(most, device="cuda")
    q = st["q"].float().view(T, Hk, G, D)[(start[:-1, None] + i[None, :]).clamp(max=T - 1)]
    q = q.permute(0, 2, 3, 1, 4).reshape(n, Hk, G * most, D)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(_softmax_scale(st)).view(n, Hk, G, most, -1)
    seen = key[None, None, :] <= (lens - count)[:, None, None] + i[None, :, None]
    s = torch.where(seen[:, None, None], s, torch.full((), -math.inf, device="cuda"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp_(s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, Hk, G * most, -1), v).view(n, Hk, G, most, D) / torch.where(total > 0, total, torch.ones_like(total))
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), t, right=True)
    st["out"].copy_(o.permute(0, 3, 1, 2, 4)[b, t - start[b]].reshape(T, H * D))
    return st["out"]


def exact(case, seed):
    """The definitions token by token and head by head, in 64 bits."""
    st = prepare(case, seed)
    if case["kind"] == "assign":
        return None
    P, Hk, D = case["page"], case["kv_heads"], case["dim"]
    H, pc = case["heads"], st["k"].shape[-1]
    k_scale, v_scale = _scales(case)
    if case["kind"] == "append":
        T = case["rows"]
        x = st["qkv"].double().view(T, H + 2 * Hk, D)
        j = torch.arange(D // 2, device="cuda")
        even, odd = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + D // 2)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["positions"].double()[:, None] * st["inv_freq"].double()[None, :])
        out = torch.empty_like(x)
        for h in range(H + 2 * Hk):
            y = x[:, h]
            gamma = st["gamma_q"] if h < H else st["gamma_k"]
            if h < H + Hk:
                if gamma is not None:
                    y = y / torch.sqrt((y * y).sum(1, keepdim=True) / D + EPS) * gamma.double()
                z = torch.complex(y[:, even].contiguous(), y[:, odd].contiguous()) * turn
                out[:, h, even], out[:, h, odd] = z.real, z.imag
            else:
                out[:, h] = y
        k, v = torch.zeros(st["k"].shape, dtype=torch.float64, device="cuda"), torch.zeros(st["v"].shape, dtype=torch.float64, device="cuda")
        top = math.inf if case["cache"] == "bf16" else 448.0
        slot = st["slots"].long()
        for h in range(Hk):
            d = torch.arange(D, device="cuda")[None, :]
            page, block, tok = slot[:, None] // P, slot[:, None] % P // 16, slot[:, None] % 16
            k[page, h, block, d // pc, tok, d % pc] = (out[:, H + h] / k_scale).clamp(-top, top)
            v[page, h, block, tok // pc, d, tok % pc] = (out[:, H + Hk + h] / v_scale).clamp(-top, top)
        return out[:, :H].reshape(T, H * D), k, v
    G = H // Hk
    q = st["q"].double().view(-1, H, D)
    out = torch.zeros_like(q)
    start, lens = st["query_start"].tolist(), st["kv_lens"].tolist()
    for b, L in enumerate(lens):
        pages = st["table"][b, :-(-L // P)].long()
        for h in range(Hk):
            k = st["k"][pages, h].double().permute(0, 1, 3, 2, 4).reshape(-1, D)[:L] * k_scale
            v = st["v"][pages, h].double().permute(0, 1, 2, 4, 3).reshape(-1, D)[:L] * v_scale
            rows = start[b + 1] - start[b]
            for g in range(G):
                s = (q[start[b]:start[b + 1], h * G + g] @ k.T) * D ** -0.5
                late = torch.arange(L, device="cuda")[None, :] > torch.arange(L - rows, L, device="cuda")[:, None]
                out[start[b]:start[b + 1], h * G + g] = torch.softmax(s.masked_fill(late, -math.inf), 1) @ v
    return out.view(-1, H * D)


def work(case):
    if case["kind"] == "assign":
        n, (new, old) = case["requests"], _lens(case, 0)
        rows = sum(new)
        need = sum(-(-(a + o) // case["page"]) - -(-o // case["page"]) for a, o in zip(new, old))
        # lengths in, lengths and starts out; each taken page read and entered; a position and a slot for each token
        return {"bytes": 4.0 * (4 * n + 2 * need + 2 * rows), "flops": 8.0 * rows}
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    size = 2 if case["cache"] == "bf16" else 1
    if case["kind"] == "append":
        T = case["rows"]
        return {"bytes": T * (2.0 * (2 * H + 2 * Hk) * D + 2.0 * Hk * D * size + 8), "flops": 8.0 * T * (H + 2 * Hk) * D}
    new, old = _lens(case, 0)
    keys = sum(a + o for a, o in zip(new, old))
    pairs = sum(a * o + a * (a + 1) // 2 for a, o in zip(new, old))
    return {"bytes": 2.0 * keys * Hk * D * size + 4.0 * sum(new) * H * D, "flops": 4.0 * pairs * H * D}
