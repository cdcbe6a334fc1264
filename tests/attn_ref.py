"""The attention block's definitions in 64 bits on the CPU, request by request, and the cache's layout element by element; shares no
code with the library."""
import numpy as np
import torch

BF16_STEP = torch.finfo(torch.bfloat16).eps / 2      # largest relative error of a rounding


def dtype_of(cache):
    return torch.bfloat16 if cache == "bf16" else torch.float8_e4m3fn


def pool_shapes(pages, kv_heads, page, dim, cache):
    pc = 8 if cache == "bf16" else 16
    return (pages, kv_heads, page // 16, dim // pc, 16, pc), (pages, kv_heads, page // 16, 16 // pc, dim, pc)


def pack(k, v, cache):
    """Tokens [pages][page][kv head][dim] to the pools' order."""
    pages, page, heads, dim = k.shape
    pc = 8 if cache == "bf16" else 16
    kp = k.reshape(pages, page // 16, 16, heads, dim // pc, pc).permute(0, 3, 1, 4, 2, 5).contiguous()
    vp = v.reshape(pages, page // 16, 16 // pc, pc, heads, dim).permute(0, 4, 1, 2, 5, 3).contiguous()
    return kp, vp


def unpack(kp, vp):
    """The pools to tokens [pages][page][kv head][dim]."""
    pages, heads, blocks, pieces, _, pc = kp.shape
    k = kp.permute(0, 2, 4, 1, 3, 5).reshape(pages, blocks * 16, heads, pieces * pc)
    v = vp.permute(0, 2, 3, 5, 1, 4).reshape(pages, blocks * 16, heads, pieces * pc)
    return k, v


def raw(t):
    """Elements as integers: 8-bit floats have few operations of their own."""
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.uint8)


def assign(new, lens, free_pages, free, table, page, rows):
    """(query_start, kv_lens, positions, slots, left, table)"""
    table = table.copy()
    width = table.shape[1]
    free = min(max(free, 0), len(free_pages))
    start, out_lens, pos, slot = [0], [], [0] * rows, [-1] * rows
    at = need_sum = taken = refused = 0
    for b, (n, length) in enumerate(zip(new, lens)):
        n, old = max(n, 0), length if length >= 0 else -1 - length
        first, last = -(-old // page), -(-(old + n) // page)
        good = last <= width and at + n <= rows
        if good:
            need_sum += last - first
            good = last == first or need_sum <= free
        if good:
            for c in range(first, last):
                table[b, c] = free_pages[free - 1 - taken]
                taken += 1
            for i in range(n):
                pos[at + i] = old + i
                slot[at + i] = table[b, (old + i) // page] * page + (old + i) % page
        refused += not good
        out_lens.append(old + n if good else -1 - old)
        at += n
        start.append(min(at, rows))
    return start, out_lens, pos, slot, [free - taken, refused], table


def append(qkv, q_heads, kv_heads, dim, gamma_q, gamma_k, eps, inv_freq, adjacent, positions):
    """(q, k, v) [rows][heads][dim] in 64 bits, and for q and k what their parts add up to in magnitude."""
    rows = qkv.shape[0]
    x = qkv.double().view(rows, -1, dim)
    q, k, v = x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]

    def norm(y, gamma):
        if gamma is None:
            return y
        ms = y.square().mean(-1, keepdim=True) + eps
        return torch.where(ms > 0, y / torch.sqrt(torch.where(ms > 0, ms, torch.ones_like(ms))), torch.zeros_like(y)) * gamma.double()

    def turn(y):
        if inv_freq is None:
            return y, y.abs()
        angle = positions.double()[:, None] * inv_freq.double()[None, :]
        i = torch.arange(dim // 2)
        ia, ib = (2 * i, 2 * i + 1) if adjacent else (i, i + dim // 2)
        a, b, c, s = y[..., ia], y[..., ib], torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        out, size = torch.empty_like(y), torch.empty_like(y)
        out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia] = size[..., ib] = a.abs() + b.abs()
        return out, size

    return turn(norm(q, gamma_q)), turn(norm(k, gamma_k)), v


def attend(q, k, v, n, scale):
    """Rows q [n][heads][dim], the last n of the keys k, v [keys][kv heads][dim]: outputs, sum p |v| / sum p, and the largest
    scale * sum |q k| of each row."""
    heads, dim = q.shape[1:]
    G = heads // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, size, score = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(n, heads, 1, dtype=torch.float64)
    L = k.shape[0]
    for h in range(heads):
        kh, vh = k[:, h // G], v[:, h // G]
        s = q[:, h] @ kh.T * scale
        late = torch.arange(L)[None, :] > torch.arange(L - n, L)[:, None]
        s = s.masked_fill(late, -np.inf)
        some = ~late.all(1)
        p = torch.softmax(s[some], 1)
        out[some, h], size[some, h] = p @ vh, p @ vh.abs()
        if some.any():
            score[some, h, 0] = (q[some, h].abs() @ kh.abs().T * abs(scale)).masked_fill(late[some], 0).amax(1)
    return out, size, score
