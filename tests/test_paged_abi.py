"""Paged cache entry points: bad host arguments are refused before any HIP call (CPU only)."""
import ctypes

import pytest

from paper_2410_23668_amd import binding as kb

A = 0x10000   # an address that is never read: every call here is refused first


def cache(**over):
    f = dict(k=A, v=A, k_scale=A, v_scale=A, dtype=kb.KL_DTYPE_E4M3, n_layers=2, n_pages=9,
             n_kv_heads=4, page_size=16, head_dim=128, device=0)
    f.update(over)
    return kb.kl_paged_cache(*[f[n] for n, _ in kb.kl_paged_cache._fields_])


def table(**over):
    f = dict(pages=A, batch=3, max_pages=5, stride=5)
    f.update(over)
    return kb.kl_page_table(*[f[n] for n, _ in kb.kl_page_table._fields_])


def rows(**over):
    f = dict(data=A, dtype=kb.KL_DTYPE_BF16, row_stride=4 * 128, head_stride=128)
    f.update(over)
    return kb.kl_rows(*[f[n] for n, _ in kb.kl_rows._fields_])


POOL = [
    (dict(c=None), kb.KL_ERR_INVALID_ARGUMENT, "cache is NULL"),
    (dict(c=cache(dtype=kb.KL_DTYPE_FP16)), kb.KL_ERR_UNSUPPORTED, "cache dtype"),
    (dict(c=cache(head_dim=96)), kb.KL_ERR_UNSUPPORTED, "head_dim"),
    (dict(c=cache(n_pages=0)), kb.KL_ERR_INVALID_ARGUMENT, "n_pages"),
    (dict(c=cache(page_size=24)), kb.KL_ERR_UNSUPPORTED, "page_size"),
    (dict(c=cache(page_size=4)), kb.KL_ERR_UNSUPPORTED, "page_size"),
    (dict(c=cache(page_size=8192)), kb.KL_ERR_UNSUPPORTED, "page_size"),
    (dict(c=cache(k=A + 8)), kb.KL_ERR_INVALID_ARGUMENT, "16-byte"),
    (dict(c=cache(v=None)), kb.KL_ERR_INVALID_ARGUMENT, "16-byte"),
    (dict(c=cache(v_scale=None)), kb.KL_ERR_INVALID_ARGUMENT, "v_scale"),
    (dict(c=cache(k_scale=A + 4)), kb.KL_ERR_INVALID_ARGUMENT, "k_scale"),
    (dict(layer=2), kb.KL_ERR_INVALID_ARGUMENT, "layer 2"),
    (dict(layer=-1), kb.KL_ERR_INVALID_ARGUMENT, "layer -1"),
    (dict(t=None), kb.KL_ERR_INVALID_ARGUMENT, "page table"),
    (dict(t=table(pages=None)), kb.KL_ERR_INVALID_ARGUMENT, "page table"),
    (dict(t=table(pages=A + 2)), kb.KL_ERR_INVALID_ARGUMENT, "page table"),
    (dict(t=table(batch=0)), kb.KL_ERR_INVALID_ARGUMENT, "batch 0"),
    (dict(t=table(stride=4)), kb.KL_ERR_INVALID_ARGUMENT, "stride 4"),
    (dict(t=table(max_pages=(1 << 26) + 1, stride=1 << 27)), kb.KL_ERR_UNSUPPORTED, "2^30"),
]
ROWS = [
    (dict(pos=A + 1), kb.KL_ERR_INVALID_ARGUMENT, "4-byte"),
    (dict(seq=A + 2), kb.KL_ERR_INVALID_ARGUMENT, "4-byte"),
    (dict(err=A + 2), kb.KL_ERR_INVALID_ARGUMENT, "4-byte"),
    (dict(pos=None), kb.KL_ERR_INVALID_ARGUMENT, "positions"),
    (dict(n=-1), kb.KL_ERR_INVALID_ARGUMENT, "rows"),
    (dict(n=1 << 31), kb.KL_ERR_INVALID_ARGUMENT, "rows"),
    (dict(seq=None, n=4), kb.KL_ERR_INVALID_ARGUMENT, "without seq"),
    (dict(k=None), kb.KL_ERR_INVALID_ARGUMENT, "k is NULL"),
    (dict(v=rows(data=None)), kb.KL_ERR_INVALID_ARGUMENT, "v is NULL"),
    (dict(k=rows(dtype=kb.KL_DTYPE_E4M3)), kb.KL_ERR_UNSUPPORTED, "k dtype"),
    (dict(k=rows(data=A + 1)), kb.KL_ERR_INVALID_ARGUMENT, "aligned"),
    (dict(v=rows(dtype=kb.KL_DTYPE_FP32, data=A + 2)), kb.KL_ERR_INVALID_ARGUMENT, "aligned"),
    (dict(v=rows(row_stride=-1)), kb.KL_ERR_INVALID_ARGUMENT, "strides"),
]


def call_rows(fn, c=cache(), layer=0, t=table(), seq=A, pos=A, n=3, k=rows(), v=rows(), err=None):
    return getattr(kb.lib(), fn)(c, layer, t, seq, pos, n, k, v, err, None)


@pytest.mark.parametrize("fn", ["kl_paged_append", "kl_paged_read"])
@pytest.mark.parametrize("over,status,msg", POOL + ROWS)
def test_append_and_read_refuse(fn, over, status, msg):
    assert call_rows(fn, **over) == status
    assert msg in kb.kl_last_error() and fn in kb.kl_last_error()


@pytest.mark.parametrize("over", [dict(row_stride=0), dict(head_stride=127), dict(head_stride=0)])
def test_read_refuses_overlapping_outputs(over):
    assert call_rows("kl_paged_read", k=rows(**over)) == kb.KL_ERR_INVALID_ARGUMENT
    assert "k strides" in kb.kl_last_error()


def call_attention(c=cache(), layer=0, t=table(), lengths=A, q=rows(), heads=8, scale=0.1,
                   window=0, out=rows(), lse=None, ws=A, ws_bytes=1 << 30, err=None):
    return kb.lib().kl_paged_attention(c, layer, t, lengths, q, heads, scale, window, out, lse, ws,
                                       ws_bytes, err, None)


@pytest.mark.parametrize("over,status,msg", POOL + [
    (dict(t=table(batch=4097)), kb.KL_ERR_UNSUPPORTED, "4096"),
    (dict(t=table(batch=4096, max_pages=1 << 18, stride=1 << 18)), kb.KL_ERR_UNSUPPORTED, "2^35"),
    (dict(heads=0), kb.KL_ERR_INVALID_ARGUMENT, "n_heads"),
    (dict(heads=10), kb.KL_ERR_INVALID_ARGUMENT, "multiple"),
    (dict(heads=4 * 17), kb.KL_ERR_UNSUPPORTED, "17 query heads"),
    (dict(lengths=None), kb.KL_ERR_INVALID_ARGUMENT, "lengths"),
    (dict(lengths=A + 2), kb.KL_ERR_INVALID_ARGUMENT, "4-byte"),
    (dict(lse=A + 2), kb.KL_ERR_INVALID_ARGUMENT, "4-byte"),
    (dict(err=A + 1), kb.KL_ERR_INVALID_ARGUMENT, "4-byte"),
    (dict(q=None), kb.KL_ERR_INVALID_ARGUMENT, "q is NULL"),
    (dict(q=rows(dtype=7)), kb.KL_ERR_UNSUPPORTED, "q dtype"),
    (dict(out=rows(head_stride=64)), kb.KL_ERR_INVALID_ARGUMENT, "out strides"),
    (dict(out=rows(row_stride=0)), kb.KL_ERR_INVALID_ARGUMENT, "out strides"),
    (dict(scale=float("nan")), kb.KL_ERR_INVALID_ARGUMENT, "scale"),
    (dict(scale=float("inf")), kb.KL_ERR_INVALID_ARGUMENT, "scale"),
    (dict(window=-1), kb.KL_ERR_INVALID_ARGUMENT, "window"),
    (dict(ws=None), kb.KL_ERR_INVALID_ARGUMENT, "workspace"),
    (dict(ws=A + 8), kb.KL_ERR_INVALID_ARGUMENT, "workspace"),
    (dict(ws_bytes=16), kb.KL_ERR_INVALID_ARGUMENT, "workspace"),
])
def test_attention_refuses(over, status, msg):
    assert call_attention(**over) == status
    assert msg in kb.kl_last_error()


@pytest.mark.parametrize("scale", [3.0e38, -3.0e38, 2.0 ** 127 * (1 + 2.0 ** -23)])
def test_attention_refuses_scales_that_overflow(scale):
    # log2(e) times such a scale may be infinite
    assert call_attention(scale=scale) == kb.KL_ERR_INVALID_ARGUMENT
    assert "2^127" in kb.kl_last_error()
    # (no GPU here: the device check that follows the arguments' may fail)
    assert call_attention(scale=2.0 ** 127, c=cache(device=77)) in (kb.KL_ERR_INVALID_ARGUMENT,
                                                                    kb.KL_ERR_HIP)
    assert "2^127" not in kb.kl_last_error()


def test_workspace_bytes():
    L = kb.lib()
    n = L.kl_paged_attention_workspace(cache(), 1)
    assert n > 0 and L.kl_paged_attention_workspace(cache(), 4096) >= n
    # (any number of heads and either type of pool: the same workspace)
    assert L.kl_paged_attention_workspace(cache(dtype=kb.KL_DTYPE_BF16, k_scale=None,
                                                v_scale=None), 1) == n
    assert L.kl_paged_attention_workspace(cache(), 0) == 0
    assert L.kl_paged_attention_workspace(cache(), 4097) == 0
    assert L.kl_paged_attention_workspace(cache(head_dim=80), 1) == 0
    assert L.kl_paged_attention_workspace(None, 1) == 0


def test_no_rows_is_no_work_but_checked():
    # (no GPU here: the device check that follows the arguments' may fail, and nothing else)
    st = call_rows("kl_paged_append", n=0, k=None, v=None, pos=None)
    assert st in (kb.KL_OK, kb.KL_ERR_HIP)
    assert call_rows("kl_paged_append", n=0, c=cache(head_dim=80)) == kb.KL_ERR_UNSUPPORTED


def test_structs_match_the_header():
    assert ctypes.sizeof(kb.kl_paged_cache) == 4 * 8 + 7 * 4 + 4
    assert ctypes.sizeof(kb.kl_page_table) == 8 + 3 * 4 + 4
    assert ctypes.sizeof(kb.kl_rows) == 8 + 8 + 2 * 8
