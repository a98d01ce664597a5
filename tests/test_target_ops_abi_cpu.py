"""Refusals and workspace queries of the rotary, latent cache and log probability entry points: host checks, no GPU work."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2509_24248_amd", "libspecexit.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libspecexit.so not built")


def plain_view(**kw):
    from paper_2509_24248_amd import binding as sx
    kv = sx.KVView()
    kv.struct_size = C.sizeof(sx.KVView)
    kv.layout, kv.dtype, kv.n_kv_heads, kv.head_dim, kv.k, kv.v, kv.l_max = 0, 1, 8, 128, 256, 512, 4096
    for n, v in kw.items():
        setattr(kv, n, v)
    return kv


def latent_view(**kw):
    from paper_2509_24248_amd import binding as sx
    kv = sx.LatentKVView()
    kv.struct_size = C.sizeof(sx.LatentKVView)
    kv.layout, kv.dtype, kv.latent_dim, kv.rope_dim, kv.c, kv.l_max = 0, 1, 512, 64, 256, 4096
    for n, v in kw.items():
        setattr(kv, n, v)
    return kv


def paged(make, **kw):
    return make(**{**dict(layout=1, page_table=256, page_size=16, max_pages_per_seq=100, n_pages=500), **kw})


def refused(sx, rc, code, text):
    assert rc == code and text in sx.last_error(), (rc, sx.last_error())


def rope(sx, desc, dtype=1, turns=256, B=2, T=3, H=4, d=128, rows=256, stride=512, out=512, out_stride=512, pos=256):
    return sx.LIB.specexit_rope(dtype, C.byref(desc), turns, B, T, H, d, rows, stride, out, out_stride, pos, None, None, 0, None)


def write(sx, kv, desc, turns=256, B=2, T=3, Hq=32, q=256, qs=4096, k=256, v=512, kvs=1024, out=1024, pos=256):
    return sx.LIB.specexit_rope_kv_write(C.byref(kv), C.byref(desc), turns, B, T, Hq, q, qs, k, v, kvs, out, pos, None, None, 0, None)


def latent_write(sx, kv, desc, turns=256, B=2, T=3, H=16, rows=256, rs=576, gain=256, eps=1e-6, q=256, qs=1024, hs=64, out=512, pos=256):
    return sx.LIB.specexit_latent_kv_write(C.byref(kv), C.byref(desc), turns, B, T, H, rows, rs, gain, eps, q, qs, hs, out, pos, None, None, 0, None)


def latent_attn(sx, kv, B=2, n_q=3, H=16, q=256, ctx=256, scale=1.0, out=512, ws=256, nbytes=1 << 34):
    return sx.LIB.specexit_latent_verify_attn(C.byref(kv), B, n_q, H, q, ctx, None, scale, out, ws, nbytes, 0, None)


def latent_compact(sx, kv, layers=2, ls=1 << 20, B=2, n_q=3, ctx=256, path=256, length=256, last=0, hidden=0, D=0, nxt=0):
    return sx.LIB.specexit_latent_kv_compact(C.byref(kv), layers, ls, B, n_q, ctx, path, length, last or None, hidden or None, D, nxt or None, 0, None)


def logprobs(sx, dtype=0, M=4, V=1000, logits=256, ld=1000, per=1, n_tok=1, token=256, lp=256, ent=256, n_top=2, top=256, ws=256, nbytes=1 << 30):
    return sx.LIB.specexit_token_logprobs(dtype, M, V, logits, ld, per, None, n_tok, token, lp, ent or None, n_top, top, None, ws, nbytes, 0, None)


BAD_ROPE = [(dict(rot_dim=0), "rot_dim"), (dict(rot_dim=7), "rot_dim"), (dict(rot_dim=258), "rot_dim"), (dict(theta=1.0), "theta"),
            (dict(theta=float("nan")), "theta"), (dict(theta=float("inf")), "theta"), (dict(amplitude=0.0), "amplitude"),
            (dict(scaling=4), "scaling"), (dict(scaling=-1), "scaling"), (dict(scaling=1, factor=0.5), "factor"), (dict(scaling=2, low=0.0), "low"),
            (dict(scaling=3, low=4.0, high=4.0), "low"), (dict(scaling=3, orig_len=0), "low")]


def test_descriptors_are_checked():
    from paper_2509_24248_amd import binding as sx
    for kw, text in BAD_ROPE:
        desc = sx.rope_desc(**{**dict(rot_dim=64), **kw})
        refused(sx, sx.LIB.specexit_rope_table(C.byref(desc), 256, None), sx.EUNSUPPORTED if "rot_dim" in kw else sx.EINVAL, text)
        for call in (lambda: rope(sx, desc), lambda: write(sx, plain_view(), desc), lambda: latent_write(sx, latent_view(), desc)):
            assert call() < 0 and text in sx.last_error()
    desc = sx.rope_desc(64)
    refused(sx, sx.LIB.specexit_rope_table(C.byref(desc), None, None), sx.EINVAL, "null")
    desc.struct_size = 4
    refused(sx, rope(sx, desc), sx.EINVAL, "ABI size")


def test_rope_refuses():
    from paper_2509_24248_amd import binding as sx
    desc = sx.rope_desc(128)
    refused(sx, rope(sx, desc, dtype=2), sx.EINVAL, "dtype")
    refused(sx, rope(sx, desc, B=0), sx.EINVAL, "B or T")
    refused(sx, rope(sx, desc, H=0), sx.EINVAL, "n_heads")
    for d in (8, 24, 520):
        refused(sx, rope(sx, desc, d=d), sx.EUNSUPPORTED, "head_dim")
    refused(sx, rope(sx, desc, d=64), sx.EINVAL, "rot_dim")
    for kw in (dict(turns=0), dict(rows=0), dict(out=0), dict(pos=0)):
        refused(sx, rope(sx, desc, **kw), sx.EINVAL, "null")
    refused(sx, rope(sx, desc, stride=511), sx.EINVAL, "stride")
    refused(sx, rope(sx, desc, out_stride=511), sx.EINVAL, "stride")
    for kw in (dict(stride=516), dict(out_stride=516), dict(rows=264), dict(out=520)):
        refused(sx, rope(sx, desc, **kw), sx.EINVAL, "aligned")
    refused(sx, rope(sx, desc, out=256, out_stride=1024), sx.EINVAL, "in place")
    refused(sx, rope(sx, desc, B=2 ** 31 - 1, T=2 ** 31 - 1), sx.EUNSUPPORTED, "more than one call")


def test_write_refuses():
    from paper_2509_24248_amd import binding as sx
    desc = sx.rope_desc(128)
    for kw, text in ((dict(struct_size=8), "ABI size"), (dict(dtype=3), "dtype"), (dict(k=0), "null"), (dict(head_dim=96), "head_dim"),
                     (dict(layout=5), "layout"), (dict(l_max=1 << 31), "entries per sequence"), (dict(v=520), "aligned")):
        assert write(sx, plain_view(**kw), desc) < 0 and text in sx.last_error(), sx.last_error()
    kv = plain_view()
    refused(sx, write(sx, plain_view(head_dim=64), desc), sx.EINVAL, "rot_dim")
    refused(sx, write(sx, kv, desc, T=0), sx.EINVAL, "B or T")
    refused(sx, write(sx, kv, desc, Hq=-1), sx.EINVAL, "heads")
    for kw in (dict(turns=0), dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(pos=0)):
        refused(sx, write(sx, kv, desc, **kw), sx.EINVAL, "null")
    refused(sx, write(sx, kv, desc, qs=4095), sx.EINVAL, "stride")
    refused(sx, write(sx, kv, desc, kvs=1023), sx.EINVAL, "stride")
    for kw in (dict(qs=4100), dict(kvs=1028), dict(q=264), dict(k=264), dict(v=264), dict(out=264)):
        refused(sx, write(sx, kv, desc, **kw), sx.EINVAL, "aligned")
    refused(sx, write(sx, kv, desc, q=1024, qs=8192, out=1024), sx.EINVAL, "in place")
    refused(sx, write(sx, kv, desc, B=1 << 20, T=1 << 20), sx.EUNSUPPORTED, "more than one call")


BAD_LATENT = [(dict(struct_size=8), "ABI size"), (dict(dtype=3), "dtype"), (dict(c=0), "null"), (dict(c=264), "aligned"), (dict(latent_dim=384), "latent_dim"),
              (dict(rope_dim=32), "rope_dim"), (dict(layout=5), "layout"), (dict(l_max=0), "l_max"), (dict(l_max=1 << 31), "entries per sequence")]
BAD_LATENT_PAGED = [(dict(page_table=0), "page_table"), (dict(page_size=24), "page_size"), (dict(n_pages=0), "empty page pool"),
                    (dict(max_pages_per_seq=0), "empty page pool"), (dict(n_pages=1 << 31), "2^35")]


def test_latent_views_are_checked():
    from paper_2509_24248_amd import binding as sx
    desc = sx.rope_desc(64)
    for make, bad in ((latent_view, BAD_LATENT), (lambda **kw: paged(latent_view, **kw), BAD_LATENT_PAGED)):
        for kw, text in bad:
            for call in (lambda kv: latent_write(sx, kv, desc), lambda kv: latent_attn(sx, kv), lambda kv: latent_compact(sx, kv)):
                assert call(make(**kw)) < 0 and text in sx.last_error(), (kw, sx.last_error())


def test_latent_write_refuses():
    from paper_2509_24248_amd import binding as sx
    kv, desc = latent_view(), sx.rope_desc(64)
    refused(sx, latent_write(sx, kv, sx.rope_desc(32)), sx.EINVAL, "rot_dim")
    refused(sx, latent_write(sx, kv, desc, B=0), sx.EINVAL, "B or T")
    refused(sx, latent_write(sx, kv, desc, H=-1), sx.EINVAL, "n_q_heads")
    for kw in (dict(turns=0), dict(rows=0), dict(pos=0), dict(q=0), dict(out=0)):
        refused(sx, latent_write(sx, kv, desc, **kw), sx.EINVAL, "null")
    for eps in (-1.0, float("nan")):
        refused(sx, latent_write(sx, kv, desc, eps=eps), sx.EINVAL, "eps")
    refused(sx, latent_write(sx, kv, desc, rs=575), sx.EINVAL, "stride")
    refused(sx, latent_write(sx, kv, desc, qs=1023), sx.EINVAL, "stride")
    refused(sx, latent_write(sx, kv, desc, hs=56), sx.EINVAL, "stride")
    for kw in (dict(rs=580), dict(gain=264), dict(rows=264), dict(qs=1028), dict(hs=68, qs=2048), dict(q=264), dict(out=264)):
        refused(sx, latent_write(sx, kv, desc, **kw), sx.EINVAL, "aligned")
    refused(sx, latent_write(sx, kv, desc, B=1 << 20, T=1 << 20), sx.EUNSUPPORTED, "more than one call")


def test_latent_attention_refuses():
    from paper_2509_24248_amd import binding as sx
    kv = latent_view()
    refused(sx, latent_attn(sx, kv, B=0), sx.EINVAL, "B < 1")
    for n_q in (0, 65):
        refused(sx, latent_attn(sx, kv, n_q=n_q), sx.EINVAL, "outside 1..64")
    for H in (0, 257, 1 << 30):
        refused(sx, latent_attn(sx, kv, H=H), sx.EUNSUPPORTED, "n_q_heads")
    refused(sx, latent_attn(sx, kv, B=1025), sx.EUNSUPPORTED, "1024 sequences")
    refused(sx, latent_attn(sx, latent_view(l_max=2)), sx.EINVAL, "fewer than the block")
    refused(sx, latent_attn(sx, latent_view(l_max=(1 << 31) - 16), B=1024), sx.EUNSUPPORTED, "can split")
    for kw in (dict(q=0), dict(ctx=0), dict(out=0)):
        refused(sx, latent_attn(sx, kv, **kw), sx.EINVAL, "null")
    refused(sx, latent_attn(sx, kv, q=264), sx.EINVAL, "aligned")
    refused(sx, latent_attn(sx, kv, out=260), sx.EINVAL, "aligned")
    for scale in (0.0, -1.0, float("nan")):
        refused(sx, latent_attn(sx, kv, scale=scale), sx.EINVAL, "scale")
    refused(sx, latent_attn(sx, kv, ws=0), sx.EWORKSPACE, "workspace")
    refused(sx, latent_attn(sx, kv, ws=128), sx.EWORKSPACE, "workspace")
    need = sx.specexit_latent_verify_attn_workspace_bytes(kv, 2, 3, 16)
    refused(sx, latent_attn(sx, kv, nbytes=need - 1), sx.EWORKSPACE, "bytes")


def test_latent_compaction_refuses():
    from paper_2509_24248_amd import binding as sx
    kv = latent_view()
    refused(sx, latent_compact(sx, kv, B=0), sx.EINVAL, "B < 1")
    refused(sx, latent_compact(sx, kv, n_q=65), sx.EINVAL, "outside 1..64")
    refused(sx, latent_compact(sx, kv, layers=0), sx.EINVAL, "n_layers")
    refused(sx, latent_compact(sx, kv, ls=8), sx.EINVAL, "stride")
    refused(sx, latent_compact(sx, kv, path=0), sx.EINVAL, "null")
    refused(sx, latent_compact(sx, kv, hidden=256, D=64), sx.EINVAL, "without last_node")
    refused(sx, latent_compact(sx, kv, hidden=256, last=256, nxt=256, D=12), sx.EINVAL, "multiple of 16")
    refused(sx, latent_compact(sx, kv, layers=70000), sx.EUNSUPPORTED, "grid")


def test_log_probabilities_refuse():
    from paper_2509_24248_amd import binding as sx
    refused(sx, logprobs(sx, dtype=5), sx.EINVAL, "dtype")
    for M in (0, 65536):
        refused(sx, logprobs(sx, M=M), sx.EINVAL, "outside 1..65535")
    refused(sx, logprobs(sx, V=0), sx.EINVAL, "V < 1")
    refused(sx, logprobs(sx, V=sx.SAMPLE_MAX_V + 1, ld=1 << 20), sx.EUNSUPPORTED, "above")
    for n in (-1, sx.LOGPROB_MAX_TOP + 1):
        refused(sx, logprobs(sx, n_top=n), sx.EUNSUPPORTED, "n_top")
    for n in (-1, sx.LOGPROB_MAX_TOK + 1):
        refused(sx, logprobs(sx, n_tok=n), sx.EUNSUPPORTED, "n_tok")
    for kw in (dict(logits=0), dict(token=0), dict(lp=0), dict(top=0)):
        refused(sx, logprobs(sx, **kw), sx.EINVAL, "null")
    refused(sx, logprobs(sx, n_tok=0, n_top=0, ent=0), sx.EINVAL, "nothing")
    refused(sx, logprobs(sx, logits=258), sx.EINVAL, "aligned")
    refused(sx, logprobs(sx, ld=999), sx.EINVAL, "row stride")
    refused(sx, logprobs(sx, per=0), sx.EINVAL, "rows_per_seq")
    refused(sx, logprobs(sx, ws=1), sx.EWORKSPACE, "workspace")
    refused(sx, logprobs(sx, nbytes=sx.specexit_token_logprobs_workspace_bytes(0, 4, 1000, 2) - 1), sx.EWORKSPACE, "bytes")


def test_a_workspace_never_shrinks():
    from paper_2509_24248_amd import binding as sx
    for n_top in (0, 5, 32):
        last = 0
        for M in list(range(1, 200)) + [1000, 65535]:
            now = sx.specexit_token_logprobs_workspace_bytes(sx.BF16, M, 151936, n_top)
            assert now >= last > -1
            last = now
        assert sx.specexit_token_logprobs_workspace_bytes(sx.BF16, 20, 151936, n_top) <= sx.specexit_token_logprobs_workspace_bytes(sx.BF16, 20, 262144, n_top)


def test_the_generic_query_agrees():
    from paper_2509_24248_amd import binding as sx
    for kv in (latent_view(), paged(latent_view), paged(latent_view, page_size=48), latent_view(latent_dim=128), latent_view(dtype=0)):
        a = sx.specexit_workspace_bytes(sx.OP_LATENT_VERIFY_ATTN, sx.latent_attn_query(kv, 16), 3, 7)
        assert a == sx.specexit_latent_verify_attn_workspace_bytes(kv, 3, 7, 16) > 0
    a = sx.specexit_workspace_bytes(sx.OP_TOKEN_LOGPROBS, sx.logprobs_query(sx.BF16, 32003, 20), 3, 7)
    assert a == sx.specexit_token_logprobs_workspace_bytes(sx.BF16, 21, 32003, 20) > 0
    assert sx.specexit_workspace_bytes(sx.OP_TOKEN_LOGPROBS, sx.logprobs_query(sx.BF16, 32003), 1 << 16, 1 << 16) == 0
    assert sx.specexit_workspace_bytes(sx.OP_ROPE, None, 4, 7) == sx.specexit_workspace_bytes(sx.OP_LATENT_KV_COMPACT, None, 4, 7) == 0
    assert sx.specexit_workspace_bytes(sx.OP_LATENT_VERIFY_ATTN, None, 4, 7) == 0
