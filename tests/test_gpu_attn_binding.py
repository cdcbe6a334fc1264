"""What the binding of the attention block refuses before it calls the library: shapes, types, strides and places of tensors.  Nothing
here reaches a kernel but the last test, whose calls have nothing to do."""
import pytest
import torch

import paper_2602_02711_amd as dmr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def b16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device=DEV)


@pytest.fixture(scope="module")
def cache():
    return dmr.KvCache.empty(4, 16, 2, 64, device=DEV)


def test_cache():
    k, v = b16(4, 2, 1, 8, 16, 8), b16(4, 2, 1, 2, 64, 8)
    c = dmr.KvCache(k, v)
    assert (c.pages, c.page_tokens, c.kv_heads, c.head_dim) == (4, 16, 2, 64)
    for bad_k, bad_v, error in ((k.cpu(), v, TypeError), (k, v.float(), TypeError), (k, v.to(torch.float8_e4m3fn), ValueError),
                                (k.transpose(0, 1), v, ValueError), (k[0], v, ValueError), (k, b16(4, 2, 1, 2, 32, 8), ValueError),
                                (k, b16(3, 2, 1, 2, 64, 8), ValueError), (b16(4, 2, 1, 4, 16, 16), v, ValueError)):
        with pytest.raises(error):
            dmr.KvCache(bad_k, bad_v)
    for args in ((4, 8, 2, 64), (4, 48, 2, 64), (4, 16, 0, 64), (4, 16, 2, 80)):
        with pytest.raises(ValueError):
            dmr.KvCache.empty(*args)


def test_assign():
    good = dict(new_tokens=i32(3), lens=i32(3), free_pages=i32(5), free_count=i32(1), block_table=i32(3, 4), page_tokens=16, rows=6)
    out = (i32(4), i32(3), i32(6), i32(6), i32(2))
    for change, error in ((dict(lens=i32(2)), ValueError), (dict(block_table=i32(2, 4)), ValueError), (dict(free_count=i32(0)), ValueError),
                          (dict(rows=-1), ValueError), (dict(new_tokens=i32(3).cpu()), TypeError), (dict(lens=i32(3).long()), TypeError),
                          (dict(block_table=i32(4, 3).t()), ValueError), (dict(free_pages=i32(10)[::2]), ValueError),
                          (dict(out=out[:4] + (i32(1),)), ValueError), (dict(out=(i32(3),) + out[1:]), ValueError),
                          (dict(out=out[:2] + (i32(6).float(),) + out[3:]), TypeError)):
        with pytest.raises(error):
            dmr.dmr_kv_assign(**{**good, **change})
    for change, status in ((dict(page_tokens=24), "unsupported"), (dict(page_tokens=0), "shape")):
        with pytest.raises(dmr.DmrError, match=status):
            dmr.dmr_kv_assign(**{**good, **change})


def test_append(cache):
    good = dict(cache=cache, qkv=b16(3, 8 * 64), q_heads=4, positions=i32(3), slots=i32(3))
    freq = torch.zeros(32, device=DEV)
    for change, error in ((dict(qkv=b16(3, 7 * 64)), ValueError), (dict(q_heads=5), ValueError), (dict(slots=i32(2)), ValueError),
                          (dict(positions=i32(4)), ValueError), (dict(gamma_q=b16(32)), ValueError), (dict(gamma_k=b16(0)), ValueError),
                          (dict(inv_freq=freq[:16]), ValueError), (dict(inv_freq=freq.double()), TypeError), (dict(qkv=b16(3, 512).float()), TypeError),
                          (dict(qkv=b16(512, 3).t()), ValueError), (dict(slots=i32(3).cpu()), TypeError), (dict(out=b16(3, 128)), ValueError),
                          (dict(out=b16(256, 3).t()), ValueError)):
        with pytest.raises(error):
            dmr.dmr_kv_append(**{**good, **change})
    with pytest.raises(dmr.DmrError, match="NULL"):            # a rotation without positions
        dmr.dmr_kv_append(**{**good, "positions": None, "inv_freq": freq})
    with pytest.raises(dmr.DmrError, match="unsupported"):
        dmr.dmr_kv_append(**good, gamma_q=b16(64), eps=-1.0)


def test_attend(cache):
    good = dict(cache=cache, q=b16(6, 256), q_heads=4, query_start=i32(4), kv_lens=i32(3), block_table=i32(3, 30), max_query=2, scale=0.1)
    for change, error in ((dict(q=b16(6, 128)), ValueError), (dict(query_start=i32(3)), ValueError), (dict(block_table=i32(2, 30)), ValueError),
                          (dict(out=b16(5, 256)), ValueError), (dict(out=b16(6, 256).float()), TypeError), (dict(kv_lens=i32(6)[::2]), ValueError),
                          (dict(block_table=i32(3, 30).long()), TypeError), (dict(q=b16(6, 256).cpu()), TypeError),
                          (dict(workspace=i32(1 << 20)), TypeError)):
        with pytest.raises(error):
            dmr.dmr_attn_paged(**{**good, **change})
    for change, status in ((dict(scale=0.0), "unsupported"), (dict(scale=float("nan")), "unsupported"), (dict(max_query=-1), "shape"),
                           (dict(workspace=torch.zeros(16, dtype=torch.uint8, device=DEV)), "workspace"),
                           (dict(q_heads=3, q=b16(6, 192)), "shape")):
        with pytest.raises(dmr.DmrError, match=status):
            dmr.dmr_attn_paged(**{**good, **change})


def test_nothing_to_do(cache):
    assert dmr.dmr_kv_append(cache, b16(0, 512), 4, None, i32(0)).shape == (0, 256)
    assert dmr.dmr_attn_paged(cache, b16(0, 256), 4, i32(3), i32(2), i32(2, 30), 1, 0.1).shape == (0, 256)
    assert (dmr.dmr_attn_paged(cache, b16(5, 256), 4, i32(1), i32(0), i32(0, 30), 1, 0.1) == 0).all()
