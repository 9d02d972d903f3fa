"""Pins of the operators' oracle (no GPU): gradients against central differences, invariants, closed forms."""
import math

import numpy as np
import pytest

from oracle import operators as O
from oracle import optim


def _difference(f, x, h=1e-5):
    """gradient of the scalar f at x by central differences: error h^2 f''' / 6 + eps |f| / h, about 1e-10"""
    g = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_turns_by_the_position_and_its_inverse_is_its_transpose(interleaved):
    rng = np.random.default_rng(0)
    freq, amp = O.rotary_frequencies(6, 100.0, "parts", 4.0, 64)
    x, y, pos = rng.normal(size=(5, 20)), rng.normal(size=(5, 20)), np.array([0, 1, -3, 70, 10 ** 6])
    r = O.rotary(x, freq, pos, 2, 10, interleaved, amplitude=amp)
    back = O.rotary(y, freq, pos, 2, 10, interleaved, inverse=True, amplitude=amp)
    assert abs((r * y).sum() - (x * back).sum()) < 1e-12
    assert np.allclose(O.rotary(r, freq, pos, 2, 10, interleaved, inverse=True, amplitude=1 / amp), x, atol=1e-12)
    assert np.array_equal(r.reshape(5, 2, 10)[..., 6:], x.reshape(5, 2, 10)[..., 6:])
    # scores depend on the distance alone
    q, k = np.repeat(x[:1], 2, 0), np.repeat(y[:1], 2, 0)
    a, b = (O.rotary(t, freq, p, 2, 10, interleaved) for t, p in ((q, [9, 109]), (k, [4, 104])))
    s = [(a[i].reshape(2, 10) * b[i].reshape(2, 10)).sum(1) for i in (0, 1)]
    assert np.allclose(s[0], s[1], atol=1e-12)


def test_rotary_scalings():
    plain, one = O.rotary_frequencies(64)
    assert one == 1.0 and plain[0] == 1.0 and math.isclose(plain[-1], 10000.0 ** (-62 / 64))
    stretched, _ = O.rotary_frequencies(64, scaling="stretched", factor=8.0)
    assert stretched[0] == 1.0 and math.isclose(stretched[-1], plain[-1] / 8)
    parts, amp = O.rotary_frequencies(64, scaling="parts", factor=8.0, length=4096)
    turns = 4096 * plain / (2 * math.pi)
    assert np.array_equal(parts[turns >= 32], plain[turns >= 32]) and np.allclose(parts[turns <= 1], plain[turns <= 1] / 8)
    assert math.isclose(amp, 0.1 * math.log(8) + 1)


@pytest.mark.parametrize("kv_heads,kv_len", [(4, None), (2, [3, 0]), (1, [5, 2])])
def test_cross_attention_gradients_against_differences(kv_heads, kv_len):
    rng = np.random.default_rng(1)
    q, k, v, g = (rng.normal(size=s) for s in ((6, 12), (10, 3 * kv_heads), (10, 3 * kv_heads), (6, 12)))
    f = lambda q, k, v: (O.cross_attention_fwd(q, k, v, 2, 4, kv_heads, kv_len)[0] * g).sum()
    dq, dk, dv = O.cross_attention_bwd(q, k, v, g, 2, 4, kv_heads, kv_len)
    assert np.allclose(dq, _difference(lambda t: f(t, k, v), q), atol=1e-8)
    assert np.allclose(dk, _difference(lambda t: f(q, t, v), k), atol=1e-8)
    assert np.allclose(dv, _difference(lambda t: f(q, k, t), v), atol=1e-8)
    if kv_len is not None and kv_len[1] == 0:
        ctx, lse = O.cross_attention_fwd(q, k, v, 2, 4, kv_heads, kv_len)
        assert not ctx[3:].any() and np.all(lse[1] == -np.inf) and not dq[3:].any() and not dk[5:].any()


@pytest.mark.parametrize("ref,ent", [(False, 0.0), (True, 0.0), (True, 0.1)])
def test_policy_loss_gradient_against_differences(ref, ent):
    rng = np.random.default_rng(2)
    T, V = 7, 11
    z, labels, adv = rng.normal(size=(T, V)) * 2, rng.integers(0, V, T), rng.normal(size=T)
    now = O.log_softmax(z)[np.arange(T), labels]
    old, r = now + 0.3 * rng.normal(size=T), now + 0.5 * rng.normal(size=T) if ref else None
    mask = np.array([1, 1, 0, 1, 1, 1, 1])
    args = dict(ref=r, mask=mask, kl_coef=0.2, ent_coef=ent, clip_low=0.2, clip_high=0.3)
    d = O.policy_loss(z, labels, old, adv, scale=0.5, **args)[4]
    assert np.allclose(d, _difference(lambda t: 0.5 * O.policy_loss(t, labels, old, adv, **args)[1].sum(), z), atol=1e-8)
    assert not d[2].any() and np.allclose(d.sum(1), 0, atol=1e-12)


@pytest.mark.parametrize("smoothing", [0.0, 0.2])
def test_preference_loss_gradient_against_differences(smoothing):
    rng = np.random.default_rng(3)
    z, labels = rng.normal(size=(12, 5)), rng.integers(0, 5, 12)
    ref, mask = rng.normal(size=4) - 4, rng.integers(0, 2, 12)
    f = lambda t: O.preference_loss(t, labels, ref, 2, 0.7, smoothing, mask)[2].sum()
    d = O.preference_loss(z, labels, ref, 2, 0.7, smoothing, mask, scale=3.0)[3]
    assert np.allclose(d, 3 * _difference(f, z), atol=1e-7)


def test_adamw_without_decay_is_adam():
    rng = np.random.default_rng(4)
    g, w, m, v = (rng.normal(size=20) for _ in range(4))
    got = O.adamw(g, w, m, v * v, 3, 1e-2, 0.9, 0.999, 1e-8, 0.0)
    want = optim.adam_step(w.copy(), g, m.copy(), (v * v).copy(), 3, 1e-2, 0.9, 0.999, 1e-8)
    assert all(np.allclose(a, b) for a, b in zip(got, want))
    decayed = O.adamw(g, w, m, v * v, 3, 1e-2, 0.9, 0.999, 1e-8, 0.5)[0]
    assert np.allclose(got[0] - decayed, 1e-2 * 0.5 * w)


def test_codes_are_what_the_type_says_and_rounding_keeps_the_mean():
    torch = pytest.importorskip("torch")
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3(codes), want, equal_nan=True)
    rng = np.random.default_rng(5)
    x = rng.normal(size=256)
    total, n = np.zeros(256), 4000
    for s in range(n):
        up, _ = O.rounding_bits(256, 7, s, 3)
        q, scale = O.quantise(x, up, False)
        total += q * scale[0]
    # a rounding has a standard deviation of at most half a step, the mean of n that over sqrt(n); six of them
    step = O.code_step(np.abs(x) / scale[0]) * scale[0]
    assert np.all(np.abs(total / n - x) <= 6 * 0.5 * step / math.sqrt(n) + 1e-12)
    q, _ = O.quantise(np.array([448.0, 1e-9, 0.0]), np.zeros(3), True)
    assert q[1] == 2.0 ** -9 and q[2] == 0.0 and q[0] == 448.0
