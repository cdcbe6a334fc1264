"""The attention block as a decoder layer uses it, between its Linears: RMSNorm and the qkv projection, pages for the new tokens, queries
and cache, attention, the output projection with the residual.  Prompts of several lengths come in as chunks, then steps of one
token, eagerly and from a captured graph that keeps its lengths, pages and free stack to itself; every step is compared with
the definition in 64 bits on the same bf16 projections."""
import numpy as np
import pytest
import torch

import paper_2602_02711_amd as dmr
from oracle import cpu_oracle as orc

import attn_ref as ref
from gpu_util import bf16_dev, quantized, u32_dev

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HIDDEN, HEADS, KV_HEADS, DIM, PAGE, EPS = 512, 8, 2, 64, 16, 1e-6
WIDTH = (HEADS + 2 * KV_HEADS) * DIM
SCALE = DIM ** -0.5


def layer(seed, N, K, copy):
    w, words, s, z = quantized(seed, N, K)
    if copy == "bf16":
        return bf16_dev(orc.f64_to_bf16(w.astype(np.float64)))
    return dmr.dmr_qlinear_create(u32_dev(words), bf16_dev(s), bf16_dev(z), 128)


def forward(copy):
    return dmr.dmr_qlinear_bf16_forward_fused if copy == "bf16" else dmr.dmr_qlinear_forward_fused


class Program:
    """A serving program's state for one layer: requests, pages, weights, and the buffers of a step of `rows` rows."""

    def __init__(self, requests, width, cache, copy, pages=None):
        self.n, self.copy = requests, copy
        self.qkv_w, self.out_w = layer(1, WIDTH, HIDDEN, copy), layer(2, HIDDEN, HEADS * DIM, copy)
        gen = torch.Generator(device=DEV).manual_seed(5)
        self.norm = (1 + 0.1 * torch.randn(HIDDEN, generator=gen, device=DEV)).bfloat16()
        self.gq, self.gk = ((1 + 0.1 * torch.randn(DIM, generator=gen, device=DEV)).bfloat16() for _ in range(2))
        self.freq = (1e4 ** (-torch.arange(0, DIM, 2, device=DEV).double() / DIM)).float()
        pages = requests * width if pages is None else pages
        scales = (1.0, 1.0) if cache == "bf16" else (0.0625, 0.0625)
        self.cache = dmr.KvCache.empty(pages, PAGE, KV_HEADS, DIM, ref.dtype_of(cache), *scales)
        for t in (self.cache.k, self.cache.v):
            ref.raw(t).fill_(0x7F)                             # NaN
        self.stack = torch.randperm(pages, generator=gen, device=DEV).int()
        self.count = torch.tensor([pages, 0], dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(requests, dtype=torch.int32, device=DEV)
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device=DEV)
        self.keys = [[] for _ in range(requests)]              # what the definition keeps: (k, v) of each chunk

    def buffers(self, rows):
        i32 = lambda m: torch.zeros(m, dtype=torch.int32, device=DEV)
        self.step = (i32(self.n + 1), self.lens, i32(rows), i32(rows), self.count)
        b = lambda w: torch.zeros(rows, w, dtype=torch.bfloat16, device=DEV)
        self.h, self.qkv, self.q, self.attn, self.y = b(HIDDEN), b(WIDTH), b(HEADS * DIM), b(HEADS * DIM), b(HIDDEN)
        self.new = i32(self.n)

    def run(self, most):
        dmr.dmr_kv_assign(self.new, self.lens, self.stack, self.count, self.table, PAGE, self.h.shape[0], out=self.step)
        start, lens, positions, slots, _ = self.step
        forward(self.copy)(self.qkv_w, dmr.DMR_PRO_RMSNORM, self.h, gamma=self.norm, eps=EPS, out=self.qkv)
        dmr.dmr_kv_append(self.cache, self.qkv, HEADS, positions, slots, self.gq, self.gk, EPS, self.freq, out=self.q)
        dmr.dmr_attn_paged(self.cache, self.q, HEADS, start, lens, self.table, most, SCALE, out=self.attn)
        forward(self.copy)(self.out_w, dmr.DMR_PRO_NONE, self.attn, residual=self.h, out=self.y)

    def check(self, new, old):
        """The step that has run brought `new` tokens to requests of `old`, and refused none."""
        rows = sum(new)
        assert self.count[1].item() == 0 and self.lens.tolist() == [a + b for a, b in zip(new, old)]
        qkv = self.qkv[:rows].cpu()
        pos = torch.cat([torch.arange(o, o + n, dtype=torch.int32) for n, o in zip(new, old)])
        assert torch.equal(self.step[2][:rows].cpu(), pos)
        (_, _), (_, _), v = ref.append(qkv, HEADS, KV_HEADS, DIM, self.gq.cpu(), self.gk.cpu(), EPS, self.freq.cpu(), False, pos)
        # queries and keys as the library rounded them (their own test holds them to the definition), values from the projection
        kc, vc = ref.unpack(self.cache.k.view(torch.uint8).cpu().view(self.cache.k.dtype).double(),
                            self.cache.v.view(torch.uint8).cpu().view(self.cache.v.dtype).double())
        kc, vc = kc.reshape(-1, KV_HEADS, DIM) * self.cache.k_scale, vc.reshape(-1, KV_HEADS, DIM) * self.cache.v_scale
        at = self.step[3][:rows].long().cpu()
        assert ((vc[at] - v).abs() <= 2.0 ** -4 * v.abs() + 2.0 ** -10).all()
        row = 0
        for b, n in enumerate(new):
            self.keys[b].append((kc[at[row:row + n]], vc[at[row:row + n]]))
            k, val = (torch.cat([c[i] for c in self.keys[b]]) for i in (0, 1))
            want, size, score = ref.attend(self.q[row:row + n].cpu().view(n, HEADS, DIM), k, val, n, SCALE)
            got = self.attn[row:row + n].cpu().double().view(n, HEADS, DIM)
            tol = (2.0 ** -8 + (DIM + 16) * 2.0 ** -22 * (1 + score)) * (size + want.abs()) * 1.01 + 2.0 ** -8 * want.abs()
            assert ((got - want).abs() <= tol).all(), (b, n)
            row += n


def hidden(p, seed, rows):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    p.h.zero_()
    p.h[:rows] = torch.randn(rows, HIDDEN, generator=gen, device=DEV).bfloat16()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("copy", ["w4", "bf16"])
def test_prompts_then_steps(cache, copy):
    p = Program(5, 12, cache, copy)
    old = [0] * 5
    for seed, new in enumerate(([37, 1, 90, 0, 16], [0, 50, 3, 15, 1], [8, 8, 8, 8, 8])):
        p.buffers(sum(new) + 3)                               # with rows of no request behind
        p.new.copy_(torch.tensor(new))
        hidden(p, seed, sum(new))
        p.run(max(new))
        torch.cuda.synchronize()
        p.check(new, old)
        old = [a + b for a, b in zip(new, old)]
    # one token each: the same step eagerly and captured
    p.buffers(5)
    p.new.fill_(1)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for step in range(9):
        hidden(p, 100 + step, 5)
        torch.cuda.synchronize()
        if step < 2:
            p.run(1)
        else:
            if step == 2:
                keep = (p.lens.clone(), p.count.clone(), p.table.clone())
                with torch.cuda.graph(graph, stream=side):
                    p.run(1)
                for t, k in zip((p.lens, p.count, p.table), keep):
                    assert torch.equal(t, k)                  # a capture runs nothing
            graph.replay()
        torch.cuda.synchronize()
        p.check([1] * 5, old)
        old = [o + 1 for o in old]
    # the output projection took what attention gave
    acc = forward(copy)(p.out_w, dmr.DMR_PRO_NONE, p.attn, residual=p.h)
    assert torch.equal(acc, p.y)


def test_a_step_without_pages_left_refuses_and_leaves_the_rest():
    p = Program(4, 8, "bf16", "w4", pages=5)
    p.buffers(80)
    new = [20, 16, 30, 14]                                     # 2 + 1 pages, then 2 of 2, then 1 of none
    p.new.copy_(torch.tensor(new))
    hidden(p, 1, 80)
    before = p.cache.k.clone().view(torch.int16)
    p.run(30)
    torch.cuda.synchronize()
    assert p.lens.tolist() == [20, 16, 30, -1] and p.count.tolist() == [0, 1]
    assert (p.step[3][66:] == -1).all() and (p.attn[66:] == 0).all() and p.attn[:66].isfinite().all()
    used = torch.unique(p.step[3][:66]).numel()
    assert used == 66
    changed = (p.cache.k.view(torch.int16) != before).view(5, KV_HEADS, 1, DIM // 8, 16, 8)
    slots = changed.any(5).any(3).any(1).reshape(-1).nonzero()[:, 0].cpu()
    assert set(slots.tolist()) <= set(p.step[3][:66].tolist())
    # pages come back (the program frees request 2), and the refused request is served as if it had not asked
    p.lens[2] = 0
    p.stack[:2] = p.table[2, :2]
    p.count[0] = 2
    p.new.copy_(torch.tensor([0, 0, 0, 14]))
    p.buffers(14)
    p.new.copy_(torch.tensor([0, 0, 0, 14]))
    hidden(p, 2, 14)
    p.run(14)
    torch.cuda.synchronize()
    assert p.lens.tolist() == [20, 16, 0, 14] and p.count.tolist() == [1, 0]
    p.keys = [[(None, None)], [(None, None)], [], []]
    at = p.step[3].long().cpu()
    kc, vc = ref.unpack(p.cache.k.cpu().double(), p.cache.v.cpu().double())
    k, v = kc.reshape(-1, KV_HEADS, DIM)[at], vc.reshape(-1, KV_HEADS, DIM)[at]
    want, size, score = ref.attend(p.q.cpu().view(14, HEADS, DIM), k, v, 14, SCALE)
    tol = (2.0 ** -8 + (DIM + 16) * 2.0 ** -22 * (1 + score)) * (size + want.abs()) * 1.01 + 2.0 ** -8 * want.abs()
    assert ((p.attn.cpu().double().view(14, HEADS, DIM) - want).abs() <= tol).all()


def test_two_calls_at_once_on_two_streams():
    """One cache read by two streams, each with its own rows, output and workspace."""
    p = Program(6, 40, "bf16", "w4")
    p.buffers(6 * 90)
    p.new.fill_(90)
    hidden(p, 3, 540)
    p.run(90)
    torch.cuda.synchronize()
    start, lens = p.step[0].clone(), p.lens.clone()
    for most, rows_of in ((90, None), (1, 1)):
        q = p.q if rows_of is None else p.q[89::90].contiguous()
        st = start if rows_of is None else torch.arange(7, dtype=torch.int32, device=DEV)
        halves = [(0, 3), (3, 6)]
        want = dmr.dmr_attn_paged(p.cache, q, HEADS, st, lens, p.table, most, SCALE)
        torch.cuda.synchronize()
        streams, outs = [torch.cuda.Stream() for _ in halves], [torch.zeros_like(want) for _ in halves]
        for _ in range(3):
            for (a, b), s, out in zip(halves, streams, outs):
                with torch.cuda.stream(s):                     # part of the batch: arrays from request a on
                    dmr.dmr_attn_paged(p.cache, q, HEADS, st[a:b + 1], lens[a:b], p.table[a:b], most, SCALE, out=out)
            torch.cuda.synchronize()
            got = outs[0] + outs[1]                            # each left the other's rows at zero
            assert ((got.double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs() + 2.0 ** -7 * want.double().abs().amax()).all()
            a_end = int(st[3])
            assert (outs[0][a_end:] == 0).all() and (outs[1][:a_end] == 0).all()


def test_tensors_that_a_call_makes_belong_to_its_stream():
    """Outputs and workspaces made by the binding are filled and reused in the order of the stream that the call names, while the current
    stream is busy and allocates the same sizes."""
    p = Program(6, 40, "bf16", "w4")
    p.buffers(6 * 90)
    p.new.fill_(90)
    hidden(p, 3, 540)
    p.run(90)
    torch.cuda.synchronize()
    args = (p.cache, p.q[89::90].contiguous(), HEADS, torch.arange(7, dtype=torch.int32, device=DEV), p.lens, p.table, 1, SCALE)
    want = dmr.dmr_attn_paged(*args)
    want_q = dmr.dmr_kv_append(p.cache, p.qkv, HEADS, p.step[2], torch.full_like(p.step[3], -1), p.gq, p.gk, EPS, p.freq)
    slow = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        for _ in range(4):
            for _ in range(3):
                slow = (slow @ slow).clamp_(-1, 1)                   # the current stream falls behind
            got = dmr.dmr_attn_paged(*args, stream=stream)
            side.synchronize()
            assert torch.equal(got, want)
            del got
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    none = torch.full_like(p.step[3], -1)
    torch.cuda.synchronize()
    q = dmr.dmr_kv_append(p.cache, p.qkv, HEADS, p.step[2], none, p.gq, p.gk, EPS, p.freq, stream=side)
    side.synchronize()
    assert torch.equal(q, want_q)
