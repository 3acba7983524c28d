"""More kernel-level entry points of token models without a GPU: what they refuse, and that both ways of calling them (_calls.so, ctypes) refuse it
alike.  Pointers are made up; every call is turned down before anything is launched."""
import ctypes

import numpy as np
import pytest

from paper_2403_08837_amd import binding as b

P = 4096          # a pointer, aligned to everything
BIG = 1 << 60     # workspace enough
INF, NAN = float("inf"), float("nan")

ROT = dict(dtype=0, qkv=P, positions=P, freqs=P, gq=P, gk=P, out=P, eps=1e-6, interleaved=0, tokens=8, heads=4, kv_heads=2, width=16, rotary=16)
ROT_B = dict(dtype=0, accumulate=0, qkv=P, positions=P, freqs=P, gq=P, gk=P, dout=P, dqkv=P, dgq=P, dgk=P, eps=1e-6, interleaved=0, ws=P, ws_bytes=8 * 16 * 8 + 256, tokens=8,
             heads=4, kv_heads=2, width=16, rotary=16)
GATED = dict(dtype=0, act=0, x=P, wg=P, wu=P, h=P, g=P, u=P, ws=P, ws_bytes=64, rows=8, inputs=16, hidden=24)
GATED_B = dict(dtype=1, act=0, x=P, wg=P, wu=P, g=P, u=P, dh=P, dx=P, dwg=P, dwu=P, ws=P, ws_bytes=4 * 8 * 24 + 1024, rows=8, inputs=16, hidden=24)
LINEAR = dict(dtype=0, act=0, x=P, w=P, bias=P, residual=P, y=P, z=P, ws=P, ws_bytes=64, rows=8, inputs=16, outputs=24)
LINEAR_B = dict(dtype=1, act=0, x=P, w=P, z=P, dy=P, dx=P, dw=P, dbias=P, ws=P, ws_bytes=2 * 8 * 24 + 4 * 24 * 8 + 1024, rows=8, inputs=16, outputs=24)
LOGP = dict(dtype=0, logits=P, ld=10, targets=P, scale=1.0, logprob=P, entropy=P, lse=P, ids=P, best=P, top=3, ws=P, ws_bytes=1 << 20, rows=4, vocab=10)
LOGP_B = dict(dtype=0, logits=P, ld=10, targets=P, scale=1.0, lse=P, entropy=P, dlogprob=P, dentropy=P, dlogits=P, rows=4, vocab=10)

REFUSED = [("cdp_k_head_norm_rotary", ROT, w) for w in (
    dict(dtype=2), dict(dtype=-1), dict(qkv=0), dict(out=0), dict(positions=0), dict(freqs=0), dict(rotary=0, gq=0, gk=0), dict(rotary=15), dict(rotary=18), dict(rotary=-2), dict(eps=0.0),
    dict(eps=-1.0), dict(eps=NAN), dict(tokens=0), dict(tokens=-1), dict(heads=0), dict(kv_heads=0), dict(width=0), dict(width=12), dict(width=136), dict(heads=4095, kv_heads=1),
    dict(qkv=P + 8), dict(out=P + 4), dict(positions=P + 2), dict(freqs=P + 1), dict(gq=P + 2), dict(gk=P + 1), dict(tokens=2 ** 31 - 1, heads=4000))]
REFUSED += [("cdp_k_head_norm_rotary_backward", ROT_B, w) for w in (
    dict(dtype=2), dict(qkv=0), dict(dout=0), dict(dqkv=0), dict(gq=0), dict(dgq=0), dict(gk=0), dict(dgk=0), dict(ws=0), dict(ws=P + 8), dict(ws_bytes=8 * 16 * 8 + 255), dict(dout=P + 8),
    dict(dqkv=P + 8), dict(dgq=P + 2), dict(dgk=P + 2), dict(eps=0.0), dict(rotary=3), dict(width=20), dict(tokens=0), dict(gq=0, dgq=0, gk=0, dgk=0, rotary=0), dict(positions=0))]
REFUSED += [("cdp_k_gated_linear", GATED, w) for w in (
    dict(dtype=2), dict(act=-1), dict(act=4), dict(x=0), dict(wg=0), dict(wu=0), dict(h=0), dict(g=0), dict(u=0), dict(rows=0), dict(rows=-4), dict(rows=(1 << 30) + 1), dict(inputs=0),
    dict(inputs=12), dict(hidden=20), dict(hidden=0), dict(inputs=(1 << 20) + 8, ws_bytes=BIG), dict(hidden=(1 << 20) + 8, ws_bytes=BIG), dict(x=P + 8), dict(wg=P + 2), dict(wu=P + 4), dict(h=P + 8), dict(g=P + 8), dict(u=P + 8), dict(ws=P + 8))]
REFUSED += [("cdp_k_gated_linear_backward", GATED_B, w) for w in (
    dict(dtype=3), dict(act=5), dict(x=0), dict(wg=0), dict(wu=0), dict(g=0), dict(u=0), dict(dh=0), dict(dwg=0), dict(dwu=0), dict(dx=0, dwg=0, dwu=0), dict(ws=0), dict(ws_bytes=4 * 8 * 24 + 1023), dict(dtype=0),
    dict(rows=0), dict(inputs=20), dict(dh=P + 8), dict(dx=P + 8), dict(dwg=P + 8), dict(dwu=P + 2), dict(ws=P + 4), dict(rows=2 ** 31 - 1, hidden=1 << 20, ws_bytes=BIG))]
REFUSED += [("cdp_k_linear", LINEAR, w) for w in (
    dict(dtype=2), dict(act=-1), dict(act=4), dict(x=0), dict(w=0), dict(y=0), dict(rows=0), dict(inputs=12), dict(outputs=20), dict(outputs=0),
    dict(inputs=(1 << 20) + 8, ws_bytes=BIG), dict(x=P + 8), dict(w=P + 2), dict(bias=P + 4), dict(residual=P + 8), dict(y=P + 8), dict(z=P + 8), dict(ws=P + 8))]
REFUSED += [("cdp_k_linear_backward", LINEAR_B, w) for w in (
    dict(dtype=3), dict(act=5), dict(z=0), dict(dy=0), dict(x=0), dict(w=0), dict(dx=0, dw=0, dbias=0), dict(ws=0), dict(ws_bytes=2 * 8 * 24 + 4 * 24 * 8 + 1023), dict(dtype=0), dict(rows=0), dict(inputs=20),
    dict(dy=P + 8), dict(dx=P + 8), dict(dw=P + 8), dict(dbias=P + 8), dict(z=P + 8), dict(ws=P + 4), dict(rows=2 ** 31 - 1, outputs=1 << 20, ws_bytes=BIG))]
REFUSED += [("cdp_k_token_logprob", LOGP, w) for w in (
    dict(dtype=2), dict(logits=0), dict(ld=9), dict(ld=2 ** 31 + 1), dict(targets=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=INF), dict(scale=NAN), dict(lse=0), dict(ids=0), dict(best=0), dict(top=-1), dict(top=11),
    dict(top=65, vocab=100, ld=100), dict(ws_bytes=(1 << 20) - 1), dict(ws=P + 8), dict(rows=0), dict(vocab=0), dict(vocab=(1 << 28) + 1, ld=1 << 29), dict(logits=P + 2), dict(dtype=1, logits=P + 1), dict(targets=P + 2),
    dict(logprob=P + 2), dict(entropy=P + 1), dict(lse=P + 2), dict(ids=P + 2), dict(best=P + 2), dict(rows=2 ** 31 - 1, ws=0))]
REFUSED += [("cdp_k_token_logprob_backward", LOGP_B, w) for w in (
    dict(dtype=2), dict(logits=0), dict(lse=0), dict(dlogits=0), dict(targets=0), dict(entropy=0), dict(dlogprob=0, dentropy=0), dict(ld=9), dict(scale=0.0), dict(scale=NAN), dict(rows=0), dict(vocab=0),
    dict(dlogits=P + 2), dict(dtype=1, dlogits=P + 1), dict(lse=P + 2), dict(entropy=P + 2), dict(dlogprob=P + 1), dict(dentropy=P + 2), dict(rows=2 ** 31 - 1))]


@pytest.mark.parametrize("name,good,change", REFUSED, ids=lambda v: v if isinstance(v, str) else ",".join("%s=%s" % p for p in v.items()) if len(v) < 7 else "")
def test_refused(name, good, change):
    """Each way of calling says CDP_EINVAL, and says which entry point."""
    args = list({**good, **change}.values()) + [0]
    with pytest.raises(b.CdpError) as e:
        getattr(b, name)(*args)
    assert e.value.code == b.CDP_EINVAL and name in str(e.value)
    assert getattr(b.lib(), name)(*args) == b.CDP_EINVAL
    assert getattr(b, "_" + name)(*args) == b.CDP_EINVAL


@pytest.mark.parametrize("name,good", [("cdp_k_head_norm_rotary", ROT), ("cdp_k_head_norm_rotary_backward", ROT_B), ("cdp_k_gated_linear", GATED), ("cdp_k_gated_linear_backward", GATED_B),
                                       ("cdp_k_linear", LINEAR), ("cdp_k_linear_backward", LINEAR_B), ("cdp_k_token_logprob", LOGP), ("cdp_k_token_logprob_backward", LOGP_B)])
def test_numbers_of_other_kinds_go_through_ctypes(name, good):
    """numpy's integers and an integer for a float are taken, or not, as ctypes does; text is not."""
    bad = dict(good, dtype=4)
    for key, v in bad.items():
        other = np.int64(v) if isinstance(v, int) else 1
        args = list({**bad, key: other}.values()) + [0]
        getattr(b, "_" + name)(*args)
        assert getattr(b, "_" + name)(*args) is None, key
        with pytest.raises((b.CdpError, ctypes.ArgumentError)):
            getattr(b, name)(*args)
    with pytest.raises(ctypes.ArgumentError):
        getattr(b, name)(*list({**bad, "dtype": "0"}.values()))


def test_in_the_list_of_exports():
    assert {name for name, _, _ in REFUSED} <= set(b.EXPORTS)


@pytest.mark.parametrize("scale", [1e-45, 9e-31, 1.1e38, 3e38])
@pytest.mark.parametrize("name,good", [("cdp_k_token_logprob", LOGP), ("cdp_k_token_logprob_backward", LOGP_B)])
def test_scales_outside_of_what_is_exact_are_refused(name, good, scale):
    args = list({**good, "scale": scale}.values()) + [0]
    with pytest.raises(b.CdpError) as e:
        getattr(b, name)(*args)
    assert e.value.code == b.CDP_EINVAL and getattr(b.lib(), name)(*args) == b.CDP_EINVAL
