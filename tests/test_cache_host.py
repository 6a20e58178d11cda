"""The paged cache's and the attention operators' refusals: every check that the
entry points make before they launch anything (no GPU is needed: the device
pointers here are never read)."""
import ctypes as C

import pytest

from paper_2306_04235_amd import mnmt

PTR, ODD = 1 << 20, (1 << 20) + 8


def pages(**kw):
    c = dict(n_layers=2, n_pages=10, page_size=16, n_kv_heads=4, d_head=64, max_pages=5)
    c.update(kw)
    return mnmt.PagesCfg(*[c[k] for k, _ in mnmt.PagesCfg._fields_])


def attn(**kw):
    c = dict(n_heads=8, kind=mnmt.ATTN_F32, causal=1, ld_q=512, ld_out=512, max_q=1, max_len=80, c_qk=0.1, c_pv=1.0)
    c.update(kw)
    return mnmt.AttnCfg(*[c[k] for k, _ in mnmt.AttnCfg._fields_])


BAD_PAGES = [dict(n_layers=0), dict(n_layers=257), dict(n_pages=0), dict(n_pages=(1 << 22) + 1), dict(page_size=8),
             dict(page_size=24), dict(page_size=512), dict(page_size=0), dict(n_kv_heads=0), dict(n_kv_heads=257),
             dict(d_head=8), dict(d_head=72), dict(d_head=144), dict(max_pages=0), dict(max_pages=(1 << 26) + 1),
             dict(n_layers=256, n_kv_heads=256, page_size=256, d_head=128)]


def refused(rc, text=None):
    assert rc == mnmt.E_INVALID_ARG
    said = mnmt.lib().mnmt_last_error().decode()
    assert said and (text is None or text in said), said


def test_sizes():
    L = mnmt.lib()
    assert L.mnmt_pages_bytes(C.byref(pages())) == 2 * 10 * 2 * 4 * 16 * 64
    assert L.mnmt_pages_bytes(C.byref(pages(n_pages=1 << 22, n_kv_heads=8))) == 2 * (1 << 22) * 2 * 8 * 16 * 64
    assert L.mnmt_pages_ws_bytes(C.byref(pages()), 7) >= 4 * (10 + 7)
    assert L.mnmt_pages_ws_bytes(C.byref(pages()), -1) == 0
    for kw in BAD_PAGES:
        assert L.mnmt_pages_bytes(C.byref(pages(**kw))) == 0, kw
        assert L.mnmt_pages_ws_bytes(C.byref(pages(**kw)), 1) == 0, kw
    assert L.mnmt_pages_bytes(None) == 0
    assert L.mnmt_attn_ws_bytes(4, 4, 8, 8, 64, 1, 40) == 0      # one pass
    assert L.mnmt_attn_ws_bytes(1, 1, 8, 8, 64, 1, 30000) > 0    # joined ranges
    big = 1 << 20
    for args in ((0, 1, 8, 8, 64, 1, big), (1, 0, 8, 8, 64, 1, big), (1, 1, 9, 8, 64, 1, big), (1, 1, 8, 8, 65, 1, big),
                 (1, 1, 8, 8, 64, -1, big), (1, 1, 8, 8, 64, 1, -1), (1, 1, 0, 1, 64, 1, big), (1, 1, 8, 0, 64, 1, big)):
        assert L.mnmt_attn_ws_bytes(*args) == 0, args


def fork(cfg=None, pool=PTR, table=PTR, lens=PTR, rows_in=4, parent=PTR, new=PTR, rows=4, table_out=2 * PTR,
         len_out=2 * PTR, info=PTR, ws=PTR, ws_bytes=1 << 20):
    return mnmt.lib().mnmt_pages_fork(C.byref(cfg or pages()), pool, table, lens, rows_in, parent, new, rows, table_out,
                                      len_out, info, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", BAD_PAGES, ids=str)
def test_page_configurations(kw):
    refused(fork(cfg=pages(**kw)))
    L, c = mnmt.lib(), pages(**kw)
    refused(L.mnmt_pages_compact(C.byref(c), PTR, PTR, PTR, 4, 2 * PTR, PTR, PTR, 1 << 20, None))
    refused(L.mnmt_pages_write(C.byref(c), PTR, 0, PTR, PTR, 4, PTR, PTR, 1 << 20, None, 4, 1, None))
    refused(L.mnmt_attn_paged(C.byref(c), C.byref(attn()), PTR, 0, PTR, PTR, 4, PTR, None, 4, PTR, PTR, 1 << 20, None))


@pytest.mark.parametrize("kw, text", [
    (dict(rows=-1), "rows"), (dict(rows_in=-1), "rows"), (dict(rows=(1 << 20) + 1), "rows"),
    (dict(rows_in=1 << 20, cfg=pages(max_pages=1 << 12)), "rows"),
    (dict(pool=None), "null"), (dict(table=None), "null"), (dict(lens=None), "null"), (dict(table_out=None), "null"),
    (dict(len_out=None), "null"), (dict(info=None), "null"), (dict(ws=None), "null"),
    (dict(pool=ODD), "aligned"), (dict(ws=ODD), "aligned"), (dict(ws_bytes=64), "smaller"),
    (dict(table_out=PTR), "overlap"), (dict(len_out=PTR), "overlap"), (dict(table_out=PTR + 16), "overlap"),
    (dict(parent=None, table_out=PTR + 16), "overlap"), (dict(parent=None, rows=5), "d_parent"),
], ids=str)
def test_fork(kw, text):
    refused(fork(**kw), text)


@pytest.mark.parametrize("kw, text", [
    (dict(rows=-1), "rows"), (dict(pool=None), "null"), (dict(table=None), "null"), (dict(lens=None), "null"),
    (dict(out=None), "null"), (dict(info=None), "null"), (dict(ws=None), "null"), (dict(pool=ODD), "aligned"),
    (dict(ws_bytes=64), "smaller"), (dict(out=PTR + 16), "overlap"),
], ids=str)
def test_compact(kw, text):
    a = dict(pool=PTR, table=PTR, lens=PTR, rows=4, out=2 * PTR, info=PTR, ws=PTR, ws_bytes=1 << 20)
    a.update(kw)
    refused(mnmt.lib().mnmt_pages_compact(C.byref(pages()), *a.values(), None), text)


@pytest.mark.parametrize("kw, text", [
    (dict(layer=-1), "layer"), (dict(layer=2), "layer"), (dict(rows=-1), "rows"), (dict(n=-1), "negative"),
    (dict(n=5), "multiple"), (dict(rows=0), "multiple"), (dict(ld=248), "ld"), (dict(ld=240), "ld"), (dict(max_q=-1), "max_q"),
    (dict(pool=None), "null"), (dict(table=None), "null"), (dict(lens=None), "null"), (dict(k=None), "null"),
    (dict(v=None), "null"), (dict(pool=ODD), "aligned"), (dict(k=ODD), "aligned"), (dict(v=ODD), "aligned"),
], ids=str)
def test_write(kw, text):
    a = dict(pool=PTR, layer=0, table=PTR, lens=PTR, rows=4, k=PTR, v=PTR, ld=768, start=None, n=4, max_q=1)
    a.update(kw)
    refused(mnmt.lib().mnmt_pages_write(C.byref(pages()), *a.values(), None), text)


BAD_ATTN = [(dict(n_heads=6), "n_heads"), (dict(n_heads=0), "n_heads"), (dict(n_heads=4100), "n_heads"),
            (dict(kind=2), "kind"), (dict(kind=-1), "kind"), (dict(ld_q=520), "ld_q"), (dict(ld_q=496), "ld_q"),
            (dict(ld_out=514), "ld_out"), (dict(ld_out=508), "ld_out"), (dict(c_qk=-1.0), "c_qk"),
            (dict(c_qk=float("nan")), "c_qk"), (dict(c_qk=float("inf")), "c_qk"), (dict(c_qk=2e30), "c_qk"),
            (dict(c_pv=float("nan")), "c_qk"), (dict(c_pv=float("inf")), "c_qk"), (dict(max_q=-1), "max_q"),
            (dict(max_len=-1), "max_q")]


@pytest.mark.parametrize("kw, text", BAD_ATTN, ids=str)
def test_attention_configurations(kw, text):
    L, c = mnmt.lib(), attn(**kw)
    refused(L.mnmt_attn_paged(C.byref(pages()), C.byref(c), PTR, 0, PTR, PTR, 4, PTR, None, 4, PTR, PTR, 1 << 20, None), text)
    c.causal = 0
    refused(L.mnmt_attn_cross(C.byref(c), 4, 64, PTR, PTR, 256, 2560, 10, PTR, 4, PTR, None, 4, PTR, PTR, 1 << 20, None), text)


@pytest.mark.parametrize("kw, text", [
    (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(rows=-1), "rows"), (dict(n=-4), "negative"), (dict(n=6), "multiple"),
    (dict(pool=None), "null"), (dict(table=None), "null"), (dict(lens=None), "null"), (dict(q=None), "null"),
    (dict(out=None), "null"), (dict(pool=ODD), "aligned"), (dict(q=ODD), "aligned"), (dict(out=ODD), "aligned"),
    (dict(cfg=attn(max_len=1 << 20), pages=pages(max_pages=1 << 12), ws_bytes=16), "workspace"),
    (dict(cfg=attn(max_len=1 << 20), pages=pages(max_pages=1 << 12), ws=None), "workspace"),
    (dict(n=1 << 30), "2^30"),
    (dict(rows=1 << 20, n=1 << 20, pages=pages(n_kv_heads=16), cfg=attn(n_heads=16, ld_q=1024, ld_out=1024)), "2^23"),
], ids=str)
def test_paged_attention(kw, text):
    a = dict(pages=pages(), cfg=attn(), pool=PTR, layer=0, table=PTR, lens=PTR, rows=4, q=PTR, start=None, n=4, out=PTR,
             ws=PTR, ws_bytes=1 << 30)
    a.update(kw)
    p, c = a.pop("pages"), a.pop("cfg")
    refused(mnmt.lib().mnmt_attn_paged(C.byref(p), C.byref(c), *a.values(), None), text)


@pytest.mark.parametrize("kw, text", [
    (dict(causal=1), "causal"), (dict(hkv=0), "n_kv_heads"), (dict(hkv=3), "n_kv_heads"), (dict(dh=40), "d_head"),
    (dict(dh=0), "d_head"), (dict(ld=264), "ld"), (dict(ld=240), "ld"), (dict(batch=100), "batch"),
    (dict(batch=-16), "batch"), (dict(S=-1), "S must"), (dict(rows=-1), "rows"), (dict(n=3), "multiple"),
    (dict(k=None), "null"), (dict(v=None), "null"), (dict(lens=None), "null"), (dict(q=None), "null"),
    (dict(out=None), "null"), (dict(k=ODD), "aligned"), (dict(v=ODD), "aligned"), (dict(q=ODD), "aligned"),
    (dict(out=ODD), "aligned"), (dict(rows=(1 << 21) + 1, n=0), "2^23"), (dict(n=1 << 30), "2^30"),
], ids=str)
def test_cross_attention(kw, text):
    a = dict(hkv=4, dh=64, k=PTR, v=PTR, ld=512, batch=5120, S=10, lens=PTR, rows=4, q=PTR, start=None, n=8, out=PTR,
             ws=None, ws_bytes=0)
    a.update({k: v for k, v in kw.items() if k != "causal"})
    refused(mnmt.lib().mnmt_attn_cross(C.byref(attn(causal=kw.get("causal", 0))), *a.values(), None), text)


def test_nothing_to_do():
    """No rows and no tokens are no error and touch nothing."""
    L, p, c = mnmt.lib(), pages(), attn(causal=0)
    assert L.mnmt_pages_write(C.byref(p), None, 0, None, None, 0, None, None, 256, None, 0, 0, None) == mnmt.OK
    assert L.mnmt_attn_paged(C.byref(p), C.byref(c), None, 0, None, None, 3, None, None, 0, None, None, 0, None) == mnmt.OK
    assert L.mnmt_attn_cross(C.byref(c), 4, 64, None, None, 256, 0, 0, None, 0, None, None, 0, None, None, 0, None) == mnmt.OK


def test_binding_refuses_what_the_kernels_would_misread():
    import torch

    pool = torch.zeros((1, 4, 2, 2, 16, 32), dtype=torch.int8)
    table, lens = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((3, 128), dtype=torch.int8)
    kv = torch.zeros((3, 5, 64), dtype=torch.int8)
    call = mnmt.mnmt_attn_paged
    for bad in (lambda: call(q.float(), pool, 0, table, lens, 1.0, 1.0), lambda: call(q[:, ::2], pool, 0, table, lens, 1.0, 1.0),
                lambda: call(q[:, :100], pool, 0, table, lens, 1.0, 1.0), lambda: call(q, pool[:, ::2], 0, table, lens, 1.0, 1.0),
                lambda: call(q, pool.float(), 0, table, lens, 1.0, 1.0), lambda: call(q, pool, 0, table.long(), lens, 1.0, 1.0),
                lambda: call(q, pool, 0, table.T, lens, 1.0, 1.0), lambda: call(q, pool, 0, table, lens[:2], 1.0, 1.0),
                lambda: call(q, pool, 0, table, lens, 1.0, 1.0, start=lens),
                lambda: mnmt.mnmt_attn_cross(q, kv, kv[:, :, ::2], lens, 32, 1.0, 1.0),
                lambda: mnmt.mnmt_attn_cross(q, kv, kv.transpose(0, 1).contiguous().transpose(0, 1), lens, 32, 1.0, 1.0),
                lambda: mnmt.mnmt_attn_cross(q, kv, kv, lens, 48, 1.0, 1.0),
                lambda: mnmt.mnmt_pages_write(pool, 0, table, lens, q, q),
                lambda: mnmt.mnmt_pages_write(pool, 0, table, lens, q[:, :64], q[:2, :64]),
                lambda: mnmt.mnmt_pages_fork(pool, table, lens, parent=lens.long()),
                lambda: mnmt.mnmt_pages_fork(pool, table, lens, new=lens[:2]),
                lambda: mnmt.mnmt_pages_compact(pool, table, lens[:1])):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("at", [0, 1, 4, 7, 8, 9, 10])
def test_binding_refuses_numbers_past_32_bits(at):
    args = [1, 1, 1, 16, 16, mnmt.ATTN_F32, 1, 16, 16, 1, 1, 1.0, 1.0]
    mnmt._attn(*args)
    args[at] += 1 << 32
    with pytest.raises(ValueError):
        mnmt._attn(*args)
