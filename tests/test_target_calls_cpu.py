"""What the binding refuses of the rotary, latent cache and log probability calls before the library sees them, and what it lets through (no GPU work)."""
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2509_24248_amd", "libspecexit.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libspecexit.so not built")


class OnDevice(torch.Tensor):                      # (for the checks behind the one of where a tensor lies; no call here gets past the library's own)
    is_cuda = True


def f(*s):
    return torch.zeros(s).as_subclass(OnDevice)


def i(*s):
    return torch.zeros(s, dtype=torch.int32).as_subclass(OnDevice)


def rejected(text, call, *args, **kw):
    with pytest.raises(AssertionError, match=text):
        call(*args, **kw)


def stopped_by_the_library(sx, text, call, *args, **kw):
    """The binding lets a call through; the library is handed something that it refuses in any call."""
    with pytest.raises(sx.SpecExitError, match=text):
        call(*args, **kw)


def turns(rot):
    return torch.zeros(rot // 2, dtype=torch.int64).as_subclass(OnDevice)


def latent(sx, B, paged):
    return sx.latent_kv_view(f(8, 16, 192), 64, i(B, 3)) if paged else sx.latent_kv_view(f(B, 48, 192), 64)


@pytest.mark.parametrize("paged", [False, True])
def test_more_sequences_than_the_cache_has(paged):
    """A view of two sequences: a third one's entries would lie behind the cache, or its pages behind the table."""
    from paper_2509_24248_amd import binding as sx
    desc, T = sx.rope_desc(64), 2
    bad = sx.rope_desc(64, theta=0.5)              # (refused by the library)
    plain = sx.kv_view(f(8, 2, 16, 64), f(8, 2, 16, 64), i(2, 3)) if paged else sx.kv_view(f(2, 2, 48, 64), f(2, 2, 48, 64))
    write = lambda B, d: sx.specexit_rope_kv_write(plain, d, turns(64), B, T, 0, None, f(B, T, 2, 64), f(B, T, 2, 64), None, i(B), stream=Null)
    rejected("has 2 sequences, 3", write, 3, desc)
    stopped_by_the_library(sx, "theta", write, 2, bad)
    kv = latent(sx, 2, paged)
    rows = lambda B, d: sx.specexit_latent_kv_write(kv, d, turns(64), B, T, 0, f(B, T, 192), None, 0.0, None, None, i(B), stream=Null)
    rejected("has 2 sequences, 3", rows, 3, desc)
    stopped_by_the_library(sx, "theta", rows, 1, bad)
    attn = lambda B: sx.specexit_latent_verify_attn(kv, B, T, 4, f(B, T, 4, 192), i(B), None, 0.0, f(B, T, 4, 128), None, stream=Null)
    rejected("has 2 sequences, 3", attn, 3)
    stopped_by_the_library(sx, "scale", attn, 2)
    compact = lambda B, layers: sx.specexit_latent_kv_compact(kv, layers, 0, B, T, i(B), i(B, T), i(B), stream=Null)
    rejected("has 2 sequences, 3", compact, 3, 1)
    stopped_by_the_library(sx, "n_layers", compact, 2, 0)


class Null:                                        # a stream by its handle
    cuda_stream = 0


def test_keys_and_values_of_one_token_may_lie_anyhow():
    """With one token of one sequence the strides of those two dimensions say nothing."""
    from paper_2509_24248_amd import binding as sx
    kv = sx.kv_view(f(1, 2, 48, 64), f(1, 2, 48, 64))
    k, v = f(1, 1, 6, 64)[:, :, :2], f(1, 1, 2, 64)
    assert k.stride() != v.stride()
    write = lambda a, b: sx.specexit_rope_kv_write(kv, sx.rope_desc(64, theta=0.5), turns(64), 1, a.shape[1], 0, None, a, b, None, i(1), stream=Null)
    stopped_by_the_library(sx, "theta", write, k, v)
    rejected("must lie alike", write, f(1, 3, 6, 64)[:, :, :2], f(1, 3, 2, 64))
    rejected("v_rows must be torch.float32", write, k, v.double())


def test_log_probabilities_without_their_tokens():
    """An output whose width is not that of what it belongs to would be left as it is, or be laid out another way."""
    from paper_2509_24248_amd import binding as sx
    M, V = 4, 100
    call = lambda **kw: sx.specexit_token_logprobs(sx.F32, M, V, f(M, V), f(M), rows_per_seq=0, stream=Null, **kw)
    rejected("logprob: \\(4, 1\\) for 0 tokens", call, logprob=f(M, 1))
    rejected("logprob: \\(4,\\) for 0 tokens", call, logprob=f(M))
    rejected("logprob: \\(4, 3\\) for 1 tokens", call, token=i(M, 1), logprob=f(M, 3))
    rejected("top_logprob: \\(4, 5\\) for 0 tokens", call, top_logprob=f(M, 5))
    rejected("top_logprob: \\(4, 5\\) for 2 tokens", call, top_token=i(M, 2), top_logprob=f(M, 5))
    for kw in (dict(token=i(M, 2), logprob=f(M, 2)), dict(token=i(M), logprob=f(M)), dict(top_token=i(M, 5)), dict(token=i(M, 0), logprob=f(M, 0)), dict(token=i(M, 1), logprob=f(2 * M, 1))):
        stopped_by_the_library(sx, "rows_per_seq", call, **kw)
