"""Refusals and workspace queries of the 8-bit cache's and the sampling entry points: host checks, no GPU work."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2509_24248_amd", "libspecexit.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libspecexit.so not built")


def view(**kw):
    from paper_2509_24248_amd import binding as sx
    kv = sx.QuantKVView()
    kv.struct_size = C.sizeof(sx.QuantKVView)
    kv.layout, kv.n_kv_heads, kv.head_dim, kv.k, kv.v, kv.k_scale, kv.v_scale, kv.l_max = 0, 8, 128, 256, 512, 768, 1024, 4096
    for n, v in kw.items():
        setattr(kv, n, v)
    return kv


def paged(**kw):
    return view(**{**dict(layout=1, page_table=256, page_size=16, max_pages_per_seq=100, n_pages=500), **kw})


BAD_VIEWS = [(dict(struct_size=8), "ABI size"), (dict(k=0), "null"), (dict(v_scale=0), "null"), (dict(k_scale=776), "aligned"),
             (dict(v=520), "aligned"), (dict(head_dim=96), "head_dim"), (dict(n_kv_heads=0), "n_kv_heads"), (dict(layout=7), "layout"),
             (dict(l_max=0), "multiple of 16"), (dict(l_max=4095), "multiple of 16"), (dict(l_max=1 << 31), "entries per sequence")]
BAD_PAGED = [(dict(page_table=0), "page_table"), (dict(page_size=8), "page_size"), (dict(page_size=24), "page_size"), (dict(n_pages=0), "empty page pool"),
             (dict(max_pages_per_seq=0), "empty page pool"), (dict(max_pages_per_seq=1 << 28), "entries per sequence")]


def write(sx, kv, dtype=1, B=2, T=3, k=256, v=512, stride=1024, pos=256, count=0):
    return sx.LIB.specexit_quant_kv_write(C.byref(kv), dtype, B, T, k, v, stride, pos, count or None, 0, None)


def attn(sx, kv, dtype=1, B=2, n_q=3, Hq=32, q=256, ctx=256, scale=1.0, out=512, ws=256, nbytes=1 << 30):
    return sx.LIB.specexit_quant_verify_attn(C.byref(kv), dtype, B, n_q, Hq, q, ctx, None, scale, out, ws, nbytes, 0, None)


def compact(sx, kv, layers=2, ls=1 << 20, ss=1 << 16, B=2, n_q=3, ctx=256, path=256, length=256, dtype=1, last=0, hidden=0, D=0, nxt=0):
    return sx.LIB.specexit_quant_kv_compact(C.byref(kv), layers, ls, ss, B, n_q, ctx, path, length, dtype, last or None, hidden or None, D, nxt or None, 0, None)


@pytest.mark.parametrize("call", [write, attn, compact])
def test_views_are_checked(call):
    from paper_2509_24248_amd import binding as sx
    for make, bad in ((view, BAD_VIEWS), (paged, BAD_PAGED)):
        for kw, text in bad:
            assert call(sx, make(**kw)) < 0 and text in sx.last_error(), (kw, sx.last_error())


def refused(sx, rc, code, text):
    assert rc == code and text in sx.last_error(), (rc, sx.last_error())


def test_write_refuses():
    from paper_2509_24248_amd import binding as sx
    kv = view()
    refused(sx, write(sx, kv, dtype=2), sx.EINVAL, "dtype")
    refused(sx, write(sx, kv, B=0), sx.EINVAL, "B or T")
    refused(sx, write(sx, kv, T=0), sx.EINVAL, "B or T")
    refused(sx, write(sx, kv, k=0), sx.EINVAL, "null")
    refused(sx, write(sx, kv, pos=0), sx.EINVAL, "null")
    refused(sx, write(sx, kv, stride=1023), sx.EINVAL, "stride")
    refused(sx, write(sx, kv, stride=1028), sx.EINVAL, "aligned")        # 2056 bytes
    refused(sx, write(sx, kv, v=520), sx.EINVAL, "aligned")
    refused(sx, write(sx, kv, B=1 << 20, T=1 << 20), sx.EUNSUPPORTED, "more than one call")


def test_attention_refuses():
    from paper_2509_24248_amd import binding as sx
    kv = view()
    refused(sx, attn(sx, kv, dtype=2), sx.EINVAL, "dtype")
    refused(sx, attn(sx, kv, B=0), sx.EINVAL, "B < 1")
    refused(sx, attn(sx, kv, n_q=0), sx.EINVAL, "outside 1..64")
    refused(sx, attn(sx, kv, n_q=65), sx.EINVAL, "outside 1..64")
    refused(sx, attn(sx, kv, Hq=30), sx.EINVAL, "multiple of n_kv_heads")
    refused(sx, attn(sx, kv, n_q=33), sx.EUNSUPPORTED, "128 query rows")
    refused(sx, attn(sx, kv, Hq=1 << 30, n_q=64), sx.EUNSUPPORTED, "128 query rows")
    refused(sx, attn(sx, kv, B=1025), sx.EUNSUPPORTED, "1024 sequences")
    refused(sx, attn(sx, view(l_max=16), n_q=17), sx.EINVAL, "fewer than the block")
    refused(sx, attn(sx, view(l_max=(1 << 31) - 16), B=1024), sx.EUNSUPPORTED, "can split")
    for kw in (dict(q=0), dict(ctx=0), dict(out=0)):
        refused(sx, attn(sx, kv, **kw), sx.EINVAL, "null")
    for scale in (0.0, -1.0, float("nan")):
        refused(sx, attn(sx, kv, scale=scale), sx.EINVAL, "scale")
    refused(sx, attn(sx, kv, ws=0), sx.EWORKSPACE, "workspace")
    refused(sx, attn(sx, kv, ws=128), sx.EWORKSPACE, "workspace")
    need = sx.specexit_quant_verify_attn_workspace_bytes(kv, sx.BF16, 2, 3, 32)
    refused(sx, attn(sx, kv, nbytes=need - 1), sx.EWORKSPACE, "bytes")


def test_compaction_refuses():
    from paper_2509_24248_amd import binding as sx
    kv = view()
    refused(sx, compact(sx, kv, B=0), sx.EINVAL, "B < 1")
    refused(sx, compact(sx, kv, n_q=65), sx.EINVAL, "outside 1..64")
    refused(sx, compact(sx, kv, layers=0), sx.EINVAL, "n_layers")
    refused(sx, compact(sx, kv, ls=8), sx.EINVAL, "strides")
    refused(sx, compact(sx, kv, ss=8), sx.EINVAL, "strides")
    refused(sx, compact(sx, kv, path=0), sx.EINVAL, "null")
    refused(sx, compact(sx, kv, hidden=256, D=64), sx.EINVAL, "without last_node")
    refused(sx, compact(sx, kv, hidden=256, last=256, nxt=256, D=12), sx.EINVAL, "multiple of 16")
    refused(sx, compact(sx, kv, hidden=256, last=256, nxt=256, D=64, dtype=9), sx.EINVAL, "dtype")
    refused(sx, compact(sx, kv, layers=70000), sx.EUNSUPPORTED, "grid")


def sample(sx, dtype=0, M=4, V=1000, logits=256, ld=1000, per=1, u=256, token=256, ws=256, nbytes=1 << 30):
    return sx.LIB.specexit_sample(dtype, M, V, logits, ld, per, None, None, None, None, u, token, None, ws, nbytes, 0, None)


def test_sampling_refuses():
    from paper_2509_24248_amd import binding as sx
    refused(sx, sample(sx, dtype=5), sx.EINVAL, "dtype")
    refused(sx, sample(sx, M=0), sx.EINVAL, "outside 1..65535")
    refused(sx, sample(sx, M=65536), sx.EINVAL, "outside 1..65535")
    refused(sx, sample(sx, V=0), sx.EINVAL, "V < 1")
    refused(sx, sample(sx, V=sx.SAMPLE_MAX_V + 1, ld=1 << 20), sx.EUNSUPPORTED, "above")
    refused(sx, sample(sx, ld=999), sx.EINVAL, "row stride")
    refused(sx, sample(sx, per=0), sx.EINVAL, "rows_per_seq")
    for kw in (dict(logits=0), dict(u=0), dict(token=0)):
        refused(sx, sample(sx, **kw), sx.EINVAL, "null")
    refused(sx, sample(sx, ws=0), sx.EWORKSPACE, "workspace")
    refused(sx, sample(sx, ws=1), sx.EWORKSPACE, "workspace")
    refused(sx, sample(sx, nbytes=sx.specexit_sample_workspace_bytes(0, 4, 1000) - 1), sx.EWORKSPACE, "bytes")


def test_the_generic_query_agrees():
    from paper_2509_24248_amd import binding as sx
    for kv in (view(), paged(), paged(page_size=48), view(head_dim=64)):
        for dtype in (sx.F32, sx.BF16):
            a = sx.specexit_workspace_bytes(sx.OP_QUANT_VERIFY_ATTN, sx.quant_attn_query(kv, dtype, 32), 3, 7)
            assert a == sx.specexit_quant_verify_attn_workspace_bytes(kv, dtype, 3, 7, 32) > 0
    a = sx.specexit_workspace_bytes(sx.OP_SAMPLE, sx.sample_query(sx.BF16, 32003), 3, 7)
    assert a == sx.specexit_sample_workspace_bytes(sx.BF16, 21, 32003) > 0
    assert sx.specexit_workspace_bytes(sx.OP_SAMPLE, sx.sample_query(sx.BF16, 32003), 1 << 16, 1 << 16) == 0
    assert sx.specexit_workspace_bytes(sx.OP_QUANT_KV_WRITE, None, 4, 7) == sx.specexit_workspace_bytes(sx.OP_QUANT_KV_COMPACT, None, 4, 7) == 0
    assert sx.specexit_workspace_bytes(sx.OP_SAMPLE, None, 4, 7) == 0
    q = sx.quant_attn_query(view(), sx.BF16, 32)
    q.struct_size = 4
    assert sx.specexit_workspace_bytes(sx.OP_QUANT_VERIFY_ATTN, q, 3, 7) == 0


@pytest.mark.parametrize("page_size", [16, 48, 64])
def test_page_tables_of_any_length_are_split(page_size):
    from paper_2509_24248_amd import binding as sx
    for pages in (1, 64, 8192, 1 << 15):
        kv = paged(page_size=page_size, max_pages_per_seq=pages, n_pages=1 << 20)
        assert sx.specexit_quant_verify_attn_workspace_bytes(kv, sx.BF16, 16, 7, 32) > 0, (pages, sx.last_error())


def test_calls_of_more_than_a_launch_are_refused():
    from paper_2509_24248_amd import binding as sx
    kv = view()
    for B, T in ((1, 2 ** 31 - 1), (2 ** 31 - 1, 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        refused(sx, write(sx, kv, B=B, T=T), sx.EUNSUPPORTED, "more than one call takes")
    refused(sx, compact(sx, kv, B=65535, layers=65535), sx.EUNSUPPORTED, "grid")
