"""The kernel-level entry points of token models without a GPU: what they refuse, and that both ways of calling them (_calls.so, ctypes) refuse it
alike.  Pointers are made up; every call is turned down before anything is launched."""
import ctypes

import numpy as np
import pytest

from paper_2403_08837_amd import binding as b

P = 4096          # a pointer, aligned to everything
BIG = 1 << 40     # workspace enough

EMBED = dict(dtype=0, backward=0, table=P, ids=P, dout=0, out=P, scale=1.0, ws=0, ws_bytes=0, rows=8, vocab=8, C=8)
EMBED_B = dict(EMBED, backward=1, table=0, dout=P, ws=P, ws_bytes=16 * 8 + 8 * 8 + 512)
NORM = dict(dtype=0, x=P, h=P, gate=P, post=P, pre=P, r=P, y=P, scale=1.0, eps=1e-6, rows=4, C=8)
NORM_B = dict(dtype=0, accumulate=0, x=P, h=P, gate=P, post=P, pre=P, dr=P, dy=P, dx=P, dh=P, dgate=P, dpost=P, dpre=P, scale=1.0, eps=1e-6, ws=P,
              ws_bytes=8 * 8 * 4 + 256, rows=4, C=8)
ATT = dict(dtype=0, backward=0, qkv=P, offsets=P, out=P, lse=P, dout=0, dqkv=0, ws=0, ws_bytes=0, tokens=8, sequences=2, heads=4, kv_heads=2, width=16, scale=0.25)
ATT_B = dict(ATT, backward=1, dout=P, dqkv=P, ws=P, ws_bytes=4 * 4 * 8 + 512)
ONE = {n: np.array([v], dtype=np.int64) for n, v in (("at", P), ("odd", P + 2), ("count", 5), ("none", 0), ("less", -1), ("lots", (1 << 40) + 1))}
CLIP = dict(dtype=0, tensors=1, grads=ONE["at"].ctypes.data, outs=ONE["at"].ctypes.data, counts=ONE["count"].ctypes.data, max_norm=1.0, norm=P, ws=P, ws_bytes=65536)

REFUSED = [("cdp_k_embedding", EMBED, w) for w in (
    dict(dtype=2), dict(dtype=-1), dict(backward=3), dict(backward=-1), dict(rows=0), dict(rows=-1), dict(vocab=0), dict(C=0), dict(C=(1 << 24) + 1), dict(scale=float("inf")), dict(scale=float("nan")), dict(table=0), dict(ids=0), dict(out=0),
    dict(table=P + 2), dict(out=P + 1), dict(ids=P + 2), dict(dtype=1, out=P + 1))]
REFUSED += [("cdp_k_embedding", EMBED_B, w) for w in (
    dict(dout=0), dict(ws=0), dict(ws_bytes=16 * 8 + 8 * 8 + 511), dict(backward=2, ws_bytes=8), dict(ws=P + 8), dict(dout=P + 2), dict(dtype=1, out=P + 2))]
REFUSED += [("cdp_k_residual_norm", NORM, w) for w in (
    dict(dtype=2), dict(x=0), dict(r=0, y=0, pre=0), dict(y=0), dict(pre=0), dict(h=0), dict(h=0, gate=0), dict(h=0, post=0), dict(rows=0), dict(C=0), dict(C=16385),
    dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("nan")), dict(x=P + 2), dict(post=P + 1), dict(dtype=1, gate=P + 1))]
REFUSED += [("cdp_k_residual_norm_backward", NORM_B, w) for w in (
    dict(dtype=2), dict(dx=0), dict(dr=0, dy=0, pre=0, dpre=0, x=0), dict(dy=0), dict(pre=0), dict(dpre=0), dict(x=0), dict(h=0), dict(dh=0), dict(dgate=0), dict(gate=0),
    dict(dpost=0), dict(post=0), dict(h=0, dh=0, post=0, dpost=0), dict(rows=0), dict(C=16385), dict(eps=0.0), dict(scale=float("inf")), dict(ws=0), dict(ws=P + 4), dict(ws_bytes=8 * 8 * 4 + 255),
    dict(dh=P + 2), dict(dpre=P + 2))]
REFUSED += [("cdp_k_attention_packed", ATT, w) for w in (
    dict(dtype=2), dict(qkv=0), dict(offsets=0), dict(out=0), dict(lse=0), dict(tokens=0), dict(sequences=0), dict(heads=0), dict(kv_heads=0), dict(heads=5), dict(kv_heads=-2),
    dict(width=0), dict(width=12), dict(width=136), dict(width=-8), dict(scale=float("nan")), dict(qkv=P + 8), dict(out=P + 4), dict(lse=P + 2), dict(offsets=P + 1), dict(heads=4095, kv_heads=1), dict(heads=2048, kv_heads=2048),
    dict(tokens=2 ** 31 - 1, heads=32))]
REFUSED += [("cdp_k_attention_packed", ATT_B, w) for w in (
    dict(dout=0), dict(dqkv=0), dict(ws=0), dict(ws_bytes=4 * 4 * 8 + 511), dict(ws=P + 8), dict(dout=P + 8), dict(dqkv=P + 8))]
REFUSED += [("cdp_k_grad_clip", CLIP, w) for w in (
    dict(dtype=2), dict(tensors=0), dict(tensors=-1), dict(grads=0), dict(counts=0), dict(norm=0), dict(ws=0), dict(ws_bytes=65535), dict(ws=P + 4), dict(norm=P + 2),
    dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(grads=ONE["none"].ctypes.data), dict(outs=ONE["none"].ctypes.data), dict(grads=ONE["odd"].ctypes.data),
    dict(outs=ONE["odd"].ctypes.data), dict(counts=ONE["less"].ctypes.data), dict(counts=ONE["lots"].ctypes.data))]

# launches that 2^32 threads would not be enough for or would just be: rows, words, the table to clear, places to merge, rows of norms, heads times tokens
REFUSED += [("cdp_k_embedding", EMBED, w) for w in (dict(rows=1 << 24, C=1025), dict(dtype=1, rows=2 ** 31 - 1, C=4096))]
REFUSED += [("cdp_k_embedding", EMBED_B, dict(ws_bytes=BIG, **w)) for w in (dict(backward=2, vocab=2 ** 31 - 1), dict(vocab=1 << 29, C=64), dict(rows=1 << 28, vocab=100))]
REFUSED += [("cdp_k_residual_norm", NORM, dict(rows=2 ** 31 - 1, C=16384))]
REFUSED += [("cdp_k_attention_packed", {**ATT, **w}, dict(tokens=2 ** 31 - 1, heads=8)) for w in (dict(), dict(dtype=1))]
REFUSED += [("cdp_k_attention_packed", {**ATT_B, **w}, dict(ws_bytes=BIG, tokens=2 ** 28, heads=8, kv_heads=4, sequences=1 << 22)) for w in (dict(), dict(dtype=1))]


@pytest.mark.parametrize("name,good,change", REFUSED, ids=lambda v: v if isinstance(v, str) else ",".join("%s=%s" % p for p in v.items()) if len(v) < 7 else "")
def test_refused(name, good, change):
    """Each way of calling says CDP_EINVAL, and says which entry point."""
    args = list({**good, **change}.values()) + [0]
    with pytest.raises(b.CdpError) as e:
        getattr(b, name)(*args)
    assert e.value.code == b.CDP_EINVAL and name in str(e.value)
    assert getattr(b.lib(), name)(*args) == b.CDP_EINVAL
    assert getattr(b, "_" + name)(*args) == b.CDP_EINVAL


@pytest.mark.parametrize("name,good", [("cdp_k_embedding", EMBED), ("cdp_k_residual_norm", NORM), ("cdp_k_residual_norm_backward", NORM_B), ("cdp_k_attention_packed", ATT),
                                       ("cdp_k_grad_clip", CLIP)])
def test_numbers_of_other_kinds_go_through_ctypes(name, good):
    """numpy's integers and an integer for a float are taken, or not, as ctypes does; text is not."""
    bad = dict(good, dtype=2)
    for key, v in bad.items():
        other = np.int64(v) if isinstance(v, int) else 1
        args = list({**bad, key: other}.values()) + [0]
        getattr(b, "_" + name)(*args)
        assert getattr(b, "_" + name)(*args) is None, key
        with pytest.raises((b.CdpError, ctypes.ArgumentError)):
            getattr(b, name)(*args)
    with pytest.raises(ctypes.ArgumentError):
        getattr(b, name)(*list({**bad, "dtype": "0"}.values()))
