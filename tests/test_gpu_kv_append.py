"""dmr_kv_append against the definition in 64 bits.

Tolerances.  Before its one rounding a query or key element is a sum of two products of (norm, gamma, cosine or sine): the norm in
fp32 is off by at most about dim 2^-24 of itself (the sum of squares, halved by the root) plus a few steps, the sine and cosine of an
angle reduced in 64 bits by 2^-18 (2^-22.3 from its 32 bits, the rest for the instruction): together below 2^-16 of |a| + |b|, the
pair's two parts.  Then half a step of the type: 2^-8 of a bf16, 2^-4 of an e4m3 and 2^-10 scales where it is subnormal."""
import pytest
import torch

import paper_2602_02711_amd as dmr

import attn_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
K_SCALE, V_SCALE = 0.05, 0.013
NEAR = 2.0 ** -16


def inv_freq(dim, theta=1e6):
    return (theta ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float()


def case(seed, rows, heads, kv_heads, dim, page, cache, norm=True, rope="halves", far=200000, pages=None):
    gen = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(rows, (heads + 2 * kv_heads) * dim, generator=gen) * 1.5).bfloat16()
    gq = (1 + 0.3 * torch.randn(dim, generator=gen)).bfloat16() if norm else None
    gk = (1 + 0.3 * torch.randn(dim, generator=gen)).bfloat16() if norm else None
    pos = torch.randint(0, far, (rows,), generator=gen, dtype=torch.int32)
    pages = pages or rows // page + 3
    slots = torch.randperm(pages * page, generator=gen)[:rows].int()
    return qkv, gq, gk, pos, slots, pages


def close(got, want, tol, where):
    off = (got.double() - want).abs() - tol
    assert torch.isfinite(got.double()).all() and (off <= 0).all(), f"{where}: {off.max():.3g} past the tolerance"


def to(t):
    return None if t is None else t.to(DEV)


def run(data, heads, kv_heads, dim, page, cache, rope, eps=1e-6, freq=None):
    qkv, gq, gk, pos, slots, pages = data
    freq = None if rope == "none" else inv_freq(dim) if freq is None else freq
    scales = (1.0, 1.0) if cache == "bf16" else (K_SCALE, V_SCALE)
    pool = dmr.KvCache.empty(pages, page, kv_heads, dim, ref.dtype_of(cache), *scales)
    for t in (pool.k, pool.v):
        ref.raw(t).fill_(0x55)
    q = dmr.dmr_kv_append(pool, to(qkv), heads, None if freq is None else to(pos), to(slots), to(gq), to(gk), eps, to(freq), rope == "adjacent")
    (wq, sq), (wk, sk), wv = ref.append(qkv, heads, kv_heads, dim, gq, gk, eps, freq, rope == "adjacent", pos)
    rows = qkv.shape[0]
    close(q.cpu().view(rows, heads, dim), wq, ref.BF16_STEP * wq.abs() + NEAR * sq, "q")
    k, v = ref.unpack(ref.raw(pool.k.cpu()), ref.raw(pool.v.cpu()))
    k, v = k.reshape(pages * page, kv_heads, dim), v.reshape(pages * page, kv_heads, dim)
    kept = (slots >= 0) & (slots < pages * page)
    at = slots[kept].long()
    other = torch.ones(pages * page, dtype=torch.bool)
    other[at] = False
    assert (k[other] == 0x55).all() and (v[other] == 0x55).all()          # no other slot was touched
    gk_, gv_ = k[at].contiguous().view(ref.dtype_of(cache)).double(), v[at].contiguous().view(ref.dtype_of(cache)).double()
    wk, sk, wv = wk[kept], sk[kept], wv[kept]
    if cache == "bf16":
        close(gk_, wk, ref.BF16_STEP * wk.abs() + NEAR * sk, "k")
        assert torch.equal(gv_, wv)
    else:
        for got, want, size, s, what in ((gk_, wk, sk, K_SCALE, "k"), (gv_, wv, wv.abs(), V_SCALE, "v")):
            want, size = (want / s).clamp(-448, 448), size / s
            close(got, want, (2.0 ** -4) * want.abs() + 2.0 ** -10 + NEAR * size, what)


SHAPES = [(1, 32, 8, 128, 64), (1, 1, 1, 64, 16), (2, 7, 1, 128, 16), (5, 16, 8, 128, 32), (33, 10, 2, 64, 128), (67, 24, 8, 64, 32),
          (130, 12, 4, 128, 256), (511, 6, 3, 64, 64), (513, 33, 3, 128, 64), (700, 8, 8, 64, 16)]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("rope", ["halves", "adjacent", "none"])
@pytest.mark.parametrize("rows,heads,kv_heads,dim,page", SHAPES)
def test_rows_to_cache(rows, heads, kv_heads, dim, page, rope, cache):
    norm = (rows + heads) % 3 != 0
    run(case(rows * 131 + heads, rows, heads, kv_heads, dim, page, cache, norm, rope), heads, kv_heads, dim, page, cache, rope)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_consecutive_tokens_from_any_place_in_a_page(cache):
    for first in (0, 3, 8, 13):
        qkv, gq, gk, pos, slots, pages = case(first, 600, 4, 2, 128, 64, cache)
        slots = torch.arange(first, first + 600, dtype=torch.int32)
        run((qkv, gq, gk, pos, slots, 12), 4, 2, 128, 64, cache, "halves")


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_rows_without_a_slot(cache):
    qkv, gq, gk, pos, slots, pages = case(4, 40, 8, 2, 64, 16, cache)
    slots[::3] = -1
    slots[1] = pages * 16
    slots[4] = 2 ** 31 - 1
    slots[7] = -2 ** 31
    run((qkv, gq, gk, pos, slots, pages), 8, 2, 64, 16, cache, "halves")
    run((qkv, gq, gk, pos, torch.full_like(slots, -1), pages), 8, 2, 64, 16, cache, "halves")


def test_one_norm_alone_zero_heads_and_far_positions():
    qkv, gq, gk, pos, slots, pages = case(9, 24, 4, 2, 128, 32, "bf16")
    qkv[3] = 0
    qkv[4, :256] = 0
    run((qkv, gq, None, pos, slots, pages), 4, 2, 128, 32, "bf16", "halves", eps=0.0)
    run((qkv, None, gk, pos, slots, pages), 4, 2, 128, 32, "bf16", "adjacent", eps=0.0)
    pos = pos + 2 ** 30
    run((qkv, gq, gk, pos, slots, pages), 4, 2, 128, 32, "bf16", "halves")
    run((qkv, gq, gk, pos, slots, pages), 4, 2, 128, 32, "bf16", "halves", freq=torch.zeros(64))


def test_values_past_the_range_of_8_bits_saturate():
    qkv, gq, gk, pos, slots, pages = case(10, 8, 2, 2, 64, 16, "e4m3", norm=False)
    run((qkv * 40, None, None, pos, slots, pages), 2, 2, 64, 16, "e4m3", "none")


@pytest.mark.parametrize("rows", [40, 700])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_elements_that_are_no_numbers_stay_so(rows, cache):
    """NaN is NaN in the cache too, and infinities are the largest of 8 bits; the elements beside them are right."""
    heads, kv_heads, dim, page = 2, 2, 64, 16
    qkv, _, _, pos, slots, pages = case(14, rows, heads, kv_heads, dim, page, cache, norm=False)
    slots = torch.arange(5, 5 + rows, dtype=torch.int32)
    odd = torch.zeros(qkv.shape, dtype=torch.bool)
    odd[::7, heads * dim::5] = True
    values = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=torch.bfloat16)
    qkv[odd] = values[torch.arange(int(odd.sum())) % 3]
    scale = 1.0 if cache == "bf16" else 0.25
    pool = dmr.KvCache.empty(pages + 1, page, kv_heads, dim, ref.dtype_of(cache), scale, scale)
    dmr.dmr_kv_append(pool, to(qkv), heads, None, to(slots))
    k, v = ref.unpack(ref.raw(pool.k.cpu()), ref.raw(pool.v.cpu()))
    at = slots.long()
    got = torch.cat([t.reshape(-1, kv_heads * dim)[at].contiguous().view(ref.dtype_of(cache)).double() for t in (k, v)], 1)
    want = qkv[:, heads * dim:].double() / scale
    if cache == "e4m3":
        want = want.clamp(-448, 448)
    assert torch.equal(got.isnan(), want.isnan())
    tol = torch.zeros_like(want) if cache == "bf16" else 2.0 ** -4 * want.abs() + 2.0 ** -10
    fine = want.isfinite()
    assert ((got - want).abs()[fine] <= tol[fine]).all()
    assert torch.equal(got[want.isinf()], want[want.isinf()])


@pytest.mark.parametrize("rows", [3, 600])
def test_cache_past_32_bits_of_bytes(rows):
    """Pages whose bytes lie past 2^32 in a pool of 4.4 GB."""
    pages, page, heads, dim = 8200, 256, 8, 128
    pool = dmr.KvCache.empty(pages, page, heads, dim)
    qkv, gq, gk, pos, _, _ = case(12, rows, 8, heads, dim, page, "bf16")
    slots = torch.arange(pages * page - rows, pages * page, dtype=torch.int32)
    dmr.dmr_kv_append(pool, to(qkv), 8, to(pos), to(slots), to(gq), to(gk), 1e-6, to(inv_freq(dim)))
    few = rows // page + 1
    k, v = ref.unpack(ref.raw(pool.k[-few:].cpu()), ref.raw(pool.v[-few:].cpu()))
    _, (wk, sk), wv = ref.append(qkv, 8, heads, dim, gq, gk, 1e-6, inv_freq(dim), False, pos)
    close(k.reshape(-1, heads, dim)[-rows:].contiguous().view(torch.bfloat16), wk, ref.BF16_STEP * wk.abs() + NEAR * sk, "k")
    assert torch.equal(v.reshape(-1, heads, dim)[-rows:].contiguous().view(torch.bfloat16).double(), wv)


@pytest.mark.parametrize("rows", [40, 700])
@pytest.mark.parametrize("rope", ["halves", "adjacent", "none"])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_normed_head_with_a_nan_is_nan_and_no_other(dim, rope, rows):
    """Its mean of squares is NaN, so all of its elements are; the same rows without it say what the other heads are."""
    heads, kv_heads, page = 4, 2, 16
    qkv, gq, gk, pos, _, pages = case(15, rows, heads, kv_heads, dim, page, "bf16")
    slots = torch.arange(rows, dtype=torch.int32)
    freq = None if rope == "none" else to(inv_freq(dim))

    def call(x):
        pool = dmr.KvCache.empty(pages, page, kv_heads, dim)
        q = dmr.dmr_kv_append(pool, to(x), heads, to(pos), to(slots), to(gq), to(gk), 1e-6, freq, rope == "adjacent")
        k, v = ref.unpack(ref.raw(pool.k.cpu()), ref.raw(pool.v.cpu()))
        k, v = (t.reshape(-1, kv_heads, dim)[:rows].contiguous().view(torch.bfloat16) for t in (k, v))
        return q.cpu().view(rows, heads, dim), k, v

    odd = qkv.clone().view(rows, heads + 2 * kv_heads, dim)
    hit = torch.zeros(rows, heads + kv_heads, dtype=torch.bool)
    hit[::3, 1] = hit[::5, heads] = hit[rows - 1, 0] = True
    for t, h in hit.nonzero().tolist():
        odd[t, h, (7 * t + h) % dim] = float("nan")
    plain, got = call(qkv), call(odd.view(rows, -1))
    hits = (hit[:, :heads], hit[:, heads:], torch.zeros(rows, kv_heads, dtype=torch.bool))
    for p, g, at in zip(plain, got, hits):
        assert g[at].isnan().all() and torch.equal(g[~at], p[~at])


@pytest.mark.parametrize("rows", [24, 700])
@pytest.mark.parametrize("power,eps", [(p, e) for p in (-133, -100, -66, -62, -51, 49, 62, 64, 120) for e in (0.0, 2.0 ** -132, 1e-6)
                                       if p > -133 or e < 1e-6])
def test_norms_of_very_small_and_very_large_heads(power, eps, rows):
    """Elements whose squares are past the ends of fp32, down to the smallest of bf16.  (2^-133 beside an eps of 1e-6 gives results with fewer
    than eight bits, which the tolerances do not count.)"""
    heads, kv_heads, dim, page = 4, 2, 128, 32
    gen = torch.Generator().manual_seed(16)
    qkv, gq, gk, pos, slots, pages = case(17, rows, heads, kv_heads, dim, page, "bf16")
    x = qkv.double() * 2.0 ** power
    x = x.view(rows, -1, dim)
    x[1::4] = 0                                                           # heads of zeros, heads of one element, and ordinary ones beside them
    x[2::4, :, 1:] = 0
    x[3::4, 1] = torch.randn(x[3::4, 1].shape, generator=gen, dtype=torch.float64)
    run((x.view(rows, -1).bfloat16(), gq, gk, pos, slots, pages), heads, kv_heads, dim, page, "bf16", "halves", eps=eps)


@pytest.mark.parametrize("rows", [40, 1024])
@pytest.mark.parametrize("scale", [0.05, 0.25, 7 / 256, 13 / 256, 15 / 256, 61 / 256, 7.0])
def test_eight_bits_of_a_value_over_its_scale(scale, rows):
    """Every finite bf16 value, or (fewer rows) those whose quotients are in range, over scales of few bits, which give ties, and others: the quotient
    in fp32, to nearest even."""
    heads, kv_heads, dim, page = 1, 1, 64, 32
    step = torch.tensor(scale, dtype=torch.float32)
    every = torch.arange(2 ** 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    every[~every.isfinite()] = 0
    if rows < 1024:
        near = (every.abs() < 448 * scale * 1.1) & (every.abs() > scale / 2048) & (every > 0)
        every = every[near][-rows * dim:]
        every = torch.cat([every, -every, torch.zeros(rows * dim, dtype=torch.bfloat16)])[:rows * dim]
    x = every.view(rows, 1, dim).expand(rows, 3, dim).reshape(rows, -1).contiguous()
    pool = dmr.KvCache.empty(rows // page + 1, page, kv_heads, dim, torch.float8_e4m3fn, scale, scale)
    dmr.dmr_kv_append(pool, to(x), heads, None, torch.arange(rows, dtype=torch.int32, device=DEV))
    want = (every.float() / step).clamp(-448, 448).to(torch.float8_e4m3fn).view(rows, dim)
    for got in ref.unpack(ref.raw(pool.k.cpu()), ref.raw(pool.v.cpu())):
        got = got.reshape(-1, dim)[:rows].contiguous().view(torch.float8_e4m3fn)
        assert torch.equal(got.double(), want.double())
