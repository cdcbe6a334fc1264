"""Refusals of the attention block's entry points: everything that the host can check is checked before the first HIP call."""
import ctypes
import os

import pytest

from paper_2602_02711_amd import binding as b

# A call that were not refused would run on addresses of no memory: never where a GPU could do that.
pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="fake addresses; the CPU alone checks refusals")

FAKE = 0x7F0000001000        # 16-byte aligned, never dereferenced by a refused call


@pytest.fixture(scope="module")
def lib():
    return b.lib()


def cache(**changes):
    fields = dict(d_k=FAKE, d_v=FAKE, pages=10, page_tokens=64, kv_heads=8, head_dim=128, type=b.DMR_KV_BF16, k_scale=1.0, v_scale=1.0)
    return ctypes.byref(b._KvCacheStruct(**{**fields, **changes}))


BAD_CACHES = [(dict(pages=0), b.DMR_ERR_SHAPE), (dict(pages=-1), b.DMR_ERR_SHAPE), (dict(pages=2 ** 25), b.DMR_ERR_SHAPE),
              (dict(page_tokens=0), b.DMR_ERR_SHAPE), (dict(page_tokens=24), b.DMR_ERR_UNSUPPORTED), (dict(page_tokens=8), b.DMR_ERR_UNSUPPORTED),
              (dict(page_tokens=512), b.DMR_ERR_UNSUPPORTED), (dict(kv_heads=0), b.DMR_ERR_SHAPE), (dict(kv_heads=3), b.DMR_ERR_SHAPE),
              (dict(head_dim=0), b.DMR_ERR_SHAPE), (dict(head_dim=96), b.DMR_ERR_UNSUPPORTED), (dict(head_dim=256), b.DMR_ERR_UNSUPPORTED),
              (dict(type=2), b.DMR_ERR_UNSUPPORTED), (dict(k_scale=0.5), b.DMR_ERR_UNSUPPORTED), (dict(v_scale=2.0), b.DMR_ERR_UNSUPPORTED),
              (dict(type=1, k_scale=0.0), b.DMR_ERR_UNSUPPORTED), (dict(type=1, v_scale=-1.0), b.DMR_ERR_UNSUPPORTED),
              (dict(type=1, v_scale=float("nan")), b.DMR_ERR_UNSUPPORTED), (dict(type=1, k_scale=float("inf")), b.DMR_ERR_UNSUPPORTED),
              (dict(type=1, k_scale=1e-40), b.DMR_ERR_UNSUPPORTED),
              (dict(d_k=None), b.DMR_ERR_NULL), (dict(d_v=None), b.DMR_ERR_NULL), (dict(d_k=FAKE + 8), b.DMR_ERR_ALIGN),
              (dict(d_v=FAKE + 4), b.DMR_ERR_ALIGN)]


def test_page_bytes(lib):
    assert lib.dmr_kv_page_bytes(64, 8, 128, b.DMR_KV_BF16) == 64 * 8 * 128 * 2
    assert lib.dmr_kv_page_bytes(16, 1, 64, b.DMR_KV_E4M3) == 16 * 64
    for bad in ((0, 8, 128, 0), (48, 8, 128, 0), (64, 0, 128, 0), (64, 8, 80, 0), (64, 8, 128, 5)):
        assert lib.dmr_kv_page_bytes(*bad) == 0


def assign(lib, requests=4, rows=8, width=3, page=16, capacity=5, **p):
    names = ["new", "lens", "stack", "count", "table", "start", "kv", "pos", "slots", "left"]
    return lib.dmr_kv_assign(requests, rows, width, page, capacity, *[p.get(n, FAKE) for n in names], None)


def test_assign(lib):
    S = b.DMR_ERR_SHAPE
    for bad, want in ((dict(requests=-1), S), (dict(requests=2 ** 20 + 1), S), (dict(rows=-1), S), (dict(rows=2 ** 22 + 1), S), (dict(width=-1), S),
                      (dict(width=2 ** 27), S), (dict(page=0), S), (dict(page=-16), S), (dict(page=40), b.DMR_ERR_UNSUPPORTED),
                      (dict(page=1024), b.DMR_ERR_UNSUPPORTED), (dict(capacity=-1), S), (dict(capacity=2 ** 31), S)):
        assert assign(lib, **bad) == want, bad
    for name in ("new", "lens", "stack", "count", "table", "start", "kv", "pos", "slots", "left"):
        assert assign(lib, **{name: None}) == b.DMR_ERR_NULL, name
        assert assign(lib, **{name: FAKE + 2}) == b.DMR_ERR_ALIGN, name


def append(lib, c=None, qkv=FAKE, rows=3, heads=32, gq=FAKE, gk=FAKE, eps=1e-6, freq=FAKE, pairs=0, pos=FAKE, slots=FAKE, q=FAKE):
    return lib.dmr_kv_append(c or cache(), qkv, rows, heads, gq, gk, eps, freq, pairs, pos, slots, q, None)


def test_append(lib):
    assert lib.dmr_kv_append(None, FAKE, 1, 32, None, None, 0.0, None, 0, None, FAKE, FAKE, None) == b.DMR_ERR_NULL
    for bad, want in BAD_CACHES:
        assert append(lib, cache(**bad)) == want, bad
    for bad, want in ((dict(rows=-1), b.DMR_ERR_SHAPE), (dict(rows=2 ** 22 + 1), b.DMR_ERR_SHAPE), (dict(heads=0), b.DMR_ERR_SHAPE),
                      (dict(heads=12), b.DMR_ERR_SHAPE), (dict(eps=-1.0), b.DMR_ERR_UNSUPPORTED), (dict(eps=float("nan")), b.DMR_ERR_UNSUPPORTED),
                      (dict(pairs=2), b.DMR_ERR_UNSUPPORTED), (dict(qkv=None), b.DMR_ERR_NULL), (dict(slots=None), b.DMR_ERR_NULL),
                      (dict(q=None), b.DMR_ERR_NULL), (dict(pos=None), b.DMR_ERR_NULL), (dict(qkv=FAKE + 8), b.DMR_ERR_ALIGN),
                      (dict(gq=FAKE + 2), b.DMR_ERR_ALIGN), (dict(gk=FAKE + 2), b.DMR_ERR_ALIGN), (dict(freq=FAKE + 4), b.DMR_ERR_ALIGN),
                      (dict(pos=FAKE + 2), b.DMR_ERR_ALIGN), (dict(slots=FAKE + 1), b.DMR_ERR_ALIGN), (dict(q=FAKE + 8), b.DMR_ERR_ALIGN),
                      (dict(rows=0), b.DMR_OK)):
        assert append(lib, **bad) == want, bad
    # an eps that no norm uses is not looked at
    assert append(lib, gq=None, gk=None, eps=-1.0, rows=0) == b.DMR_OK


def attend(lib, c=None, q=FAKE, rows=8, heads=32, requests=8, start=FAKE, lens=FAKE, table=FAKE, width=4, most=1, scale=0.1, out=FAKE, ws=FAKE,
           ws_bytes=1 << 40):
    return lib.dmr_attn_paged(c or cache(), q, rows, heads, requests, start, lens, table, width, most, scale, out, ws, ws_bytes, None)


def test_attend(lib):
    assert lib.dmr_attn_paged(None, FAKE, 1, 32, 1, FAKE, FAKE, FAKE, 1, 1, 0.1, FAKE, FAKE, 1 << 30, None) == b.DMR_ERR_NULL
    for bad, want in BAD_CACHES:
        assert attend(lib, cache(**bad)) == want, bad
    S, U, N, A = b.DMR_ERR_SHAPE, b.DMR_ERR_UNSUPPORTED, b.DMR_ERR_NULL, b.DMR_ERR_ALIGN
    for bad, want in ((dict(rows=-1), S), (dict(rows=2 ** 22 + 1), S), (dict(requests=-1), S), (dict(requests=2 ** 20 + 1), S), (dict(width=0), S),
                      (dict(width=2 ** 26), S), (dict(most=-1), S), (dict(heads=33), S), (dict(heads=-8), S), (dict(scale=float("inf")), U),
                      (dict(scale=float("nan")), U), (dict(scale=0.0), U),
                      (dict(scale=-0.1), U), (dict(scale=1e-40), U), (dict(q=None), N), (dict(start=None), N), (dict(lens=None), N), (dict(table=None), N),
                      (dict(out=None), N), (dict(q=FAKE + 8), A), (dict(out=FAKE + 2), A), (dict(ws=FAKE + 8), A), (dict(start=FAKE + 2), A),
                      (dict(lens=FAKE + 1), A), (dict(table=FAKE + 3), A), (dict(rows=0), b.DMR_OK), (dict(requests=0), b.DMR_OK),
                      (dict(most=0), b.DMR_OK)):
        assert attend(lib, **bad) == want, bad
    # with a long table, the plan is the one that the query answers for
    for rows, requests, most in ((1, 1, 1), (8, 8, 1), (300, 1, 300), (40, 8, 5)):
        need = lib.dmr_attn_paged_workspace_bytes(rows, requests, 32, 8, 128, most)
        assert need > 0
        assert attend(lib, rows=rows, requests=requests, most=most, width=2 ** 20, ws_bytes=need - 1) == b.DMR_ERR_WORKSPACE
        assert attend(lib, rows=rows, requests=requests, most=most, width=2 ** 20, ws=None) == b.DMR_ERR_WORKSPACE


def test_workspace_query(lib):
    need = lib.dmr_attn_paged_workspace_bytes
    assert need(8192, 1, 32, 8, 128, 8192) == 0                  # enough tiles without a split
    for bad in ((0, 1, 32, 8, 128, 1), (1, 0, 32, 8, 128, 1), (1, 1, 0, 8, 128, 1), (1, 1, 32, 0, 128, 1), (1, 1, 32, 5, 128, 1), (1, 1, 32, 8, 80, 1),
                (1, 1, 32, 8, 128, 0), (2 ** 23, 1, 32, 8, 128, 1), (1, 2 ** 21, 32, 8, 128, 1)):
        assert need(*bad) == 0
    # never more than fits a card by orders of magnitude, whatever the batch
    assert need(2 ** 20, 2 ** 20, 32, 8, 128, 1) < 64 << 30


def test_binding_checks_before_the_library():
    torch = pytest.importorskip("torch")
    with pytest.raises(TypeError):
        b.KvCache(torch.zeros(1, 1, 1, 16, 16, 8, dtype=torch.bfloat16), torch.zeros(1, 1, 1, 2, 128, 8, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        b.KvCache.empty(4, 16, 2, 128, torch.float16, device="cpu")
    with pytest.raises(ValueError):
        b.KvCache.empty(4, 24, 2, 128, device="cpu")


def aligned(n):
    return -(-n // 256) * 256


# rows to a key head, and requests x key heads up to where a batch is not split any more; then batches of tiles up to one for each CU
FEW = [(255, 32, 8, 128, 1), (255, 64, 8, 128, 4), (512, 12, 3, 128, 8), (512, 3, 3, 64, 17), (1, 32, 1, 128, 1), (511, 32, 4, 64, 2), (200, 7, 1, 128, 3)]
TILES = [(31, 32, 8, 128, 30), (1, 32, 8, 128, 1024), (1, 1, 1, 64, 33), (63, 16, 4, 64, 30), (40, 8, 1, 128, 50), (7, 64, 2, 128, 20)]


@pytest.mark.parametrize("requests,heads,kv_heads,dim,most", FEW + TILES)
def test_workspaces_are_as_large_as_the_largest_plan(lib, requests, heads, kv_heads, dim, most):
    """The query answers for any table and either cache type: what the parts of the batch can need at most, no less than any call asks for, and
    not much more."""
    rows = requests * most
    need = lib.dmr_attn_paged_workspace_bytes(rows, requests, heads, kv_heads, dim, most)
    to_a_head = most * (heads // kv_heads)
    if to_a_head <= 32:
        tile, items = (16 if to_a_head <= 16 else 32), requests + max(1024 // kv_heads, 2 * requests)
    else:
        tile, tiles = 128, min(requests * -(-to_a_head // 128), rows * (heads // kv_heads) // 128 + requests)
        items = tiles * min(32, max(1, 512 // (tiles * kv_heads)))
        assert items > tiles                               # these cases are split
    parts = items * kv_heads * tile
    assert need == aligned(parts * dim * 4) + aligned(parts * 8) + (requests * 8 if tile < 128 else 0)
    # a call that passes every check finds no GPU here
    for kind in (b.DMR_KV_BF16, b.DMR_KV_E4M3):
        for width in (1, 2, 4, 5, 8, 16, 33, 64, 100, 300, 1000, 5000, 2 ** 20, 2 ** 24):
            c = cache(kv_heads=kv_heads, head_dim=dim, type=kind)
            got = attend(lib, c, rows=rows, heads=heads, requests=requests, width=width, most=most, ws_bytes=need)
            assert got == b.DMR_ERR_HIP, (width, got)
