"""The formulas that the GPU tests of more token operators compare against: their gradients against differences of their values, in 64 bits.  No GPU."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import test_gpu_more_token_kernels as k  # noqa: E402

STEP = 1e-6


def against_differences(value, inputs, grads, weights):
    """`value(inputs)` weighted by `weights`, along random directions: a central difference is off by STEP^2 times a third derivative, and by 2^-53 / STEP of
    the values, 1e-10 of them."""
    g = torch.Generator()
    g.manual_seed(0)
    for name, x in inputs.items():
        v = torch.randn(x.shape, generator=g, dtype=torch.float64)
        ends = [sum(float((out * w).sum()) for out, w in zip(value({**inputs, name: x + s * STEP * v}), weights)) for s in (1, -1)]
        slope, want = (ends[0] - ends[1]) / (2 * STEP), float((grads[name] * v).sum())
        assert abs(slope - want) < 1e-7 * (1 + abs(want)) + 1e-9 * abs(ends[0]) / STEP * 1e-3, (name, slope, want)


@pytest.mark.parametrize("case", [(5, 4, 2, 16, 16, False, "qk", 50), (3, 2, 1, 24, 8, True, "qk", 9), (4, 3, 3, 8, 6, False, "q", 7), (4, 1, 1, 16, 16, True, "", 30), (2, 2, 2, 8, 0, False, "qk", 0)])
def test_rotary(case):
    T, H, K, W, R, inter, gammas, far = case
    qkv, pos, freqs, gq, gk, dout = k.rotary_inputs(case, k.F32, 3)
    inputs = {"qkv": qkv.double()}
    if gq is not None:
        inputs["gq"] = gq.double()
    if gk is not None:
        inputs["gk"] = gk.double()

    def reference(q):
        return k.rotary_reference(q["qkv"], pos, freqs, q.get("gq"), q.get("gk"), dout, k.EPS, inter, T, H, K, W, R)
    r = reference(inputs)
    against_differences(lambda q: [reference(q)["out"]], inputs, {"qkv": r["dqkv"], "gq": r["dgq"], "gk": r["dgk"]}, [dout.double()])


@pytest.mark.parametrize("act", range(4))
def test_activations(act):
    g = k.randn(1, 50, scale=3)
    w = k.randn(2, 50)
    against_differences(lambda q: [k.act_of(act, q["g"])[0]], {"g": g}, {"g": w * k.act_of(act, g)[1]}, [w])


def test_gated_and_linear():
    x, wg, wu, dh = k.randn(1, 7, 9), k.randn(2, 5, 9), k.randn(3, 5, 9), k.randn(4, 7, 5)
    for act in range(4):
        def value(q):
            return [k.act_of(act, q["x"] @ q["wg"].t())[0] * (q["x"] @ q["wu"].t())]
        g, u = x @ wg.t(), x @ wu.t()
        a, da = k.act_of(act, g)
        dg, du = dh * u * da, dh * a
        against_differences(value, dict(x=x, wg=wg, wu=wu), dict(x=dg @ wg + du @ wu, wg=dg.t() @ x, wu=du.t() @ x), [dh])
        bias = k.randn(5, 5)
        z = x @ wg.t() + bias
        dz = dh * k.act_of(act, z)[1]
        against_differences(lambda q: [k.act_of(act, q["x"] @ q["w"].t() + q["b"])[0]], dict(x=x, w=wg, b=bias), dict(x=dz @ wg, w=dz.t() @ x, b=dz.sum(0)), [dh])


def test_logprob():
    scale, rows, V = 0.7, 5, 11
    logits, dl, de = k.randn(1, rows, V, scale=2), k.randn(2, rows), k.randn(3, rows)
    targets = torch.from_numpy(np.random.default_rng(0).integers(0, V, rows))

    def value(q):
        r = k.logprob_reference(q["logits"], targets, scale, 0)
        return [r["logp"].gather(1, targets[:, None])[:, 0], r["entropy"]]
    r = k.logprob_reference(logits, targets, scale, 0)
    one = torch.zeros_like(logits).scatter_(1, targets[:, None], 1.0)
    d = scale * (dl[:, None] * (one - r["prob"]) - de[:, None] * r["prob"] * (r["logp"] + r["entropy"][:, None]))
    against_differences(value, {"logits": logits}, {"logits": d}, [dl, de])
