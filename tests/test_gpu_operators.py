"""Operators around the stage against the 64-bit oracle (GPU only), element by element.

u is half a step of the storage type (finfo.eps / 2), e that of fp32 (2^-24).  Bounds are worked out from the formulas: one
rounding of the result to the storage type, the roundings that a kernel makes to operands of matrix instructions (u each,
of the terms they enter), and for sums in 32 bits n e times the sum of the terms' magnitudes, n the number of terms."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2204_12013_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2204_12013_amd import binding
    return binding


def unit(dtype):
    return torch.finfo(torch.bfloat16 if dtype == 1 else torch.float32).eps / 2


def draw(rng, shape, dtype, scale=1.0):
    """values of the storage type, as float64, and the tensor that holds them"""
    a = synth.round_to_storage((rng.standard_normal(shape) * scale).astype(np.float32), dtype)
    return a.astype(np.float64), torch.from_numpy(a).to(torch.bfloat16 if dtype == 1 else torch.float32).to(DEV)


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV)


def host(t):
    return t.detach().double().cpu().numpy()


def within(got, want, bound, label):
    got = host(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape, label
    err = np.abs(got - want)
    assert np.all(np.isfinite(err)), label
    worst = np.max(err / np.maximum(bound, 1e-300)) if err.size else 0.0
    assert worst <= 1.0, "%s: %.2f of the bound" % (label, worst)


def strided(t, extra, fill=7.0):
    """the same matrix as a view with `extra` columns behind every row, and what holds it"""
    whole = torch.full((t.shape[0], t.shape[1] + extra), fill, dtype=t.dtype, device=t.device)
    whole[:, :t.shape[1]] = t
    return whole[:, :t.shape[1]], whole


# ---- rotary positions -----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T,heads,d,rot,extra", [
    (1, 1, 2, 2, 0), (1, 32, 64, 64, 16), (7, 5, 80, 20, 3), (33, 3, 6, 2, 0), (130, 25, 64, 64, 1600), (300, 2, 128, 128, 0),
    (5, 192, 128, 64, 8), (19, 4, 18, 18, 1), (64, 1, 512, 512, 0), (2, 3, 33, 16, 0)])
def test_rotary(B, dtype, T, heads, d, rot, extra):
    rng = np.random.default_rng(T + heads)
    freq, amp = B.bk_rotary_frequencies(rot, 10000.0, "parts", 8.0, 64)
    f, _ = O.rotary_frequencies(rot, 10000.0, "parts", 8.0, 64)
    x, xd = draw(rng, (T, heads * d), dtype)
    pos = rng.integers(-10 ** 6, 10 ** 6, T).astype(np.int32)
    for interleaved in (False, True):
        for inverse in (False, True):
            for p in (None, pos):
                want = O.rotary(x, f, np.arange(T) % 5 if p is None else p, heads, d, interleaved, inverse, amp)
                # an angle at most pi in 32 bits 1.2e-7 off, its sine and cosine 2 units more, times the amplitude and a product
                # and a sum of two terms, each rounded: 5e-7 of |a| + |b|; 64-bit products of far positions add 2^-53 of the angle
                a = np.abs(O.rotary(x, f * 0, np.zeros(T), heads, d, interleaved)).reshape(T, heads, d)[..., :rot]
                pair = (a[..., 0::2] + a[..., 1::2]).repeat(2, -1) if interleaved else np.tile(a[..., :rot // 2] + a[..., rot // 2:], 2)
                bound = np.zeros((T, heads, d))
                bound[..., :rot] = pair * amp * (5e-7 + 2e-16 * 10 ** 6)
                bound = bound.reshape(T, -1) + unit(dtype) * np.abs(want) + 1e-40
                keep = None if p is None else torch.from_numpy(p).to(DEV)
                args = dict(pos=keep, seq=5, interleaved=interleaved, inverse=inverse, amplitude=amp)
                xs, whole = strided(xd, extra)
                y, y_whole = strided(torch.zeros_like(xd), 2 * extra)
                B.bk_rotary(xs, freq, y, heads, d, **args)
                within(y, want, bound, "rotary")
                assert torch.equal(xs, xd) and (not extra or bool((y_whole[:, heads * d:] == 7).all()))
                B.bk_rotary(xs, freq, xs, heads, d, **args)                  # in place: the same bits, nothing beside it
                assert torch.equal(xs, y) and (not extra or bool((whole[:, heads * d:] == 7).all()))


def test_rotary_in_place_on_the_queries_and_keys_of_a_packed_projection(B):
    T, heads, d = 12, 4, 64
    rng = np.random.default_rng(0)
    x, xd = draw(rng, (T, 3 * heads * d), 1)
    freq, _ = B.bk_rotary_frequencies(d)
    values = xd[:, 2 * heads * d:].clone()
    B.bk_rotary(xd, freq, xd, 2 * heads, d, seq=6)
    want = O.rotary(x[:, :2 * heads * d], O.rotary_frequencies(d)[0], np.arange(T) % 6, 2 * heads, d)
    within(xd[:, :2 * heads * d], want, unit(1) * np.abs(want) + 1e-5, "packed")
    assert torch.equal(xd[:, 2 * heads * d:], values)


# ---- attention over an encoder's states -------------------------------------------------------------

def attention_bounds(q, k, v, g, ctx, lse, batch, heads, kv_heads, kv_len, u, low):
    """bounds of ctx, lse, dq, dk, dv.  low: half a step of the type that probabilities and dS have as operands."""
    d = q.shape[1] // heads
    out = [np.zeros(t.shape) for t in (q, q, k, v)]
    b_lse = np.zeros(lse.shape)
    for b, h, rq, rk, cq, ck in O._heads(q, k, v, batch, heads, kv_heads, kv_len):
        if rk.start == rk.stop:
            continue
        n, m = rk.stop - rk.start, rq.stop - rq.start
        mags = np.abs(q[rq, cq]) @ np.abs(k[rk, ck]).T / math.sqrt(d)
        z = q[rq, cq] @ k[rk, ck].T / math.sqrt(d)
        p = np.exp(z - lse[b, h][:, None])
        # scores: d products and sums and the scale; exponent and running maximum a few units of their size; sum of n terms
        dz = E * ((d + 4) * mags + 4 * np.abs(z) + 4 * np.abs(z).max(1, keepdims=True) + 8)
        b_lse[b, h] = (p * dz).sum(1) + E * (n + 8 + 2 * np.abs(lse[b, h])) + dz.max(1)
        rel = dz + b_lse[b, h][:, None]                                     # of a probability
        dp, av = p * (rel + low), np.abs(v[rk, ck])
        out[0][rq, cq] = dp @ av + E * (n + 8) * (p @ av) + u * np.abs(ctx[rq, cq])
        if g is None:
            continue
        go = np.abs(g[rq, cq])
        s = 1 / math.sqrt(d)
        delta = (g[rq, cq] * ctx[rq, cq]).sum(1, keepdims=True)
        b_delta = (go * (out[0][rq, cq] + E * (d + 2) * np.abs(ctx[rq, cq]))).sum(1, keepdims=True)
        gv = g[rq, cq] @ v[rk, ck].T
        ds = p * (gv - delta)
        b_ds = p * (rel * np.abs(gv - delta) + b_delta + E * (d + 4) * (go @ av.T + np.abs(delta))) + low * np.abs(ds)
        b_ds = b_ds * (1 + 4 * low)
        ak, aq = np.abs(k[rk, ck]), np.abs(q[rq, cq])
        out[1][rq, cq] = s * (b_ds @ ak + E * (n + 8) * (np.abs(ds) @ ak)) + u * np.abs(s * (ds @ k[rk, ck]))
        out[2][rk, ck] += s * (b_ds.T @ aq + E * (m * heads // kv_heads + 8) * (np.abs(ds).T @ aq))
        out[3][rk, ck] += dp.T @ go + E * (m * heads // kv_heads + 8) * (p.T @ go)
    return out[0], b_lse, out[1], out[2], out[3]


def run_attention(B, rng, dtype, impl, batch, sq, sk, heads, kv_heads, d, kv_len, extra=0, garbage=None):
    q, qd = draw(rng, (batch * sq, heads * d), dtype, 1.3)
    kv, kvd = draw(rng, (batch * sk, 2 * kv_heads * d), dtype)
    g, gd = draw(rng, (batch * sq, heads * d), dtype, 0.1)
    k, v = kv[:, :kv_heads * d], kv[:, kv_heads * d:]
    n = None if kv_len is None else torch.tensor(kv_len, dtype=torch.int32, device=DEV)
    if garbage is not None:
        for b in range(batch):
            kvd[b * sk + min(max(kv_len[b], 0), sk):(b + 1) * sk] = garbage
    qd, gd = (strided(t, extra)[0] for t in (qd, gd))
    kvd = strided(kvd, extra)[0]
    kd, vd = kvd[:, :kv_heads * d], kvd[:, kv_heads * d:]
    ctx, ctx_whole = strided(torch.empty_like(gd.contiguous()), extra)
    dq, dq_whole = strided(torch.empty_like(gd.contiguous()), extra)
    dkv, dkv_whole = strided(torch.full((batch * sk, 2 * kv_heads * d), 3.0, dtype=qd.dtype, device=DEV), extra)
    lse = torch.empty(batch, heads, sq, device=DEV)
    B.bk_cross_attention_fwd(qd, kd, vd, ctx, lse, batch, heads, kv_heads, kv_len=n, impl=impl)
    B.bk_cross_attention_bwd(qd, kd, vd, ctx, lse, gd, dq, dkv[:, :kv_heads * d], dkv[:, kv_heads * d:], batch, heads, kv_heads,
                             kv_len=n, impl=impl)
    want_ctx, want_lse = O.cross_attention_fwd(q, k, v, batch, heads, kv_heads, kv_len)
    want = O.cross_attention_bwd(q, k, v, g, batch, heads, kv_heads, kv_len)
    u = unit(dtype)
    low = u if dtype == 1 and impl != 1 else E
    b_ctx, b_lse, b_dq, b_dk, b_dv = attention_bounds(q, k, v, g, want_ctx, want_lse, batch, heads, kv_heads, kv_len, u, low)
    within(ctx, want_ctx, b_ctx, "ctx")
    got_lse = host(lse)
    empty = np.isinf(want_lse)
    assert np.array_equal(np.isneginf(got_lse), empty)
    within(np.where(empty, 0, got_lse), np.where(empty, 0, want_lse), b_lse, "lse")
    within(dq, want[0], b_dq, "dq")
    within(dkv[:, :kv_heads * d], want[1], b_dk + u * np.abs(want[1]), "dk")
    within(dkv[:, kv_heads * d:], want[2], b_dv + u * np.abs(want[2]), "dv")
    if extra:
        for whole in (ctx_whole, dq_whole, dkv_whole):
            assert bool((whole[:, -extra:] == 7).all())
    return ctx, lse, dq, dkv


SHAPES = [
    # batch, sq, sk, heads, kv_heads, d, key lengths
    (1, 1, 1, 1, 1, 64, None), (2, 1, 700, 4, 2, 64, [700, 3]), (1, 1, 2050, 8, 1, 128, None), (2, 3, 65, 2, 2, 128, [0, 65]),
    (2, 130, 77, 4, 4, 64, [77, 64]), (1, 200, 333, 6, 2, 128, None), (3, 65, 129, 2, 1, 64, [1, 128, 129]),
    (1, 1000, 64, 4, 1, 64, None), (1, 700, 1, 2, 2, 128, None), (2, 33, 600, 3, 3, 64, [599, -4]), (1, 5, 640, 12, 1, 64, [1000])]


@pytest.mark.parametrize("batch,sq,sk,heads,kv_heads,d,kv_len", SHAPES)
@pytest.mark.parametrize("dtype,impl", [(0, 0), (1, 2), (1, 1)])
def test_cross_attention(B, dtype, impl, batch, sq, sk, heads, kv_heads, d, kv_len):
    run_attention(B, np.random.default_rng(sq + sk), dtype, impl, batch, sq, sk, heads, kv_heads, d, kv_len)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d", [1, 2, 7, 32, 36, 80, 96, 100, 127])
def test_cross_attention_any_head_size(B, dtype, d):
    run_attention(B, np.random.default_rng(d), dtype, 0, 2, 37, 150, 4, 2, d, [150, 45])


@pytest.mark.parametrize("dtype,extra", [(0, 4), (0, 1), (1, 8), (1, 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_cross_attention_rows_with_other_columns_behind(B, dtype, extra, d):
    run_attention(B, np.random.default_rng(extra), dtype, 0, 2, 70, 200, 4, 2, d, [200, 90], extra=extra)


@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), -3e38])
@pytest.mark.parametrize("dtype,impl", [(0, 0), (1, 2), (1, 1)])
def test_keys_behind_the_length_are_not_read(B, dtype, impl, garbage):
    run_attention(B, np.random.default_rng(3), dtype, impl, 3, 40, 130, 4, 2, 64, [0, 70, 129], garbage=garbage)
    run_attention(B, np.random.default_rng(4), dtype, impl, 2, 1, 900, 2, 1, 128, [300, 0], garbage=garbage)


def test_cross_attention_is_reproducible_and_takes_any_stream(B):
    rng = np.random.default_rng(9)
    first = run_attention(B, rng, 1, 0, 2, 3, 1500, 4, 2, 64, [1500, 700])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run_attention(B, np.random.default_rng(9), 1, 0, 2, 3, 1500, 4, 2, 64, [1500, 700])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_cross_attention_of_the_own_states_is_self_attention(B):
    """one length, one key head per query head: the framework's attention over a packed qkv"""
    batch, S, heads, d = 2, 300, 4, 64
    _, qkv = draw(np.random.default_rng(5), (batch * S, 3 * heads * d), 1)
    ctx, other = (torch.empty(batch * S, heads * d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lse, lse2 = (torch.empty(batch, heads, S, device=DEV) for _ in range(2))
    B.bk_attention_fwd(qkv, ctx, lse, batch, S, heads, False)
    H = heads * d
    B.bk_cross_attention_fwd(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], other, lse2, batch, heads)
    # both round the same probabilities to bf16 and the result once
    assert float((ctx.float() - other.float()).abs().max()) <= 4 * unit(1) * float(ctx.float().abs().max())
    assert float((lse - lse2).abs().max()) <= 16 * E * float(lse.abs().max())


# ---- losses ---------------------------------------------------------------------------------------

def loss_inputs(rng, T, V, dtype, extra):
    z, zd = draw(rng, (T, V), dtype, 2.5)
    labels = rng.integers(0, V, T)
    zs, whole = strided(zd, extra)
    now = O.log_softmax(z)[np.arange(T), labels]
    return z, zs, labels, torch.from_numpy(labels.astype(np.int32)).to(DEV), now


def logp_bounds(z):
    """(error of logp and lse per token, relative error of a probability per element)"""
    t = np.abs(z - z.max(1, keepdims=True))
    p = np.exp(O.log_softmax(z))
    # exponents: two roundings of t log2 e; a thread's sum of at most 128 terms or, of longer rows, V / 1024, then 6 + 16 more
    s = E * (4 * (p * t).sum(1) + max(128, z.shape[1] / 1024 * 2) + 30)
    b = s + E * (4 + np.abs(z).max(1) + 2 * np.abs(np.log(np.exp(-t).sum(1))))
    return b, E * 4 * (t + 2) + b[:, None]


VOCABS = [1, 5, 100, 2047, 2048, 4100, 8191, 16384, 32003, 50257, 65541, 140001]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("with_ref,ent,masked,extra", [(True, 0.01, True, 0), (False, 0.0, False, 3)])
def test_policy_loss(B, dtype, V, with_ref, ent, masked, extra):
    rng = np.random.default_rng(V)
    T = 6
    z, zd, labels, lab, now = loss_inputs(rng, T, V, dtype, extra)
    old, adv = (np.float32(now + 0.2 * rng.normal(size=T)).astype(np.float64), np.float32(rng.normal(size=T)).astype(np.float64))
    ref = np.float32(now + 0.4 * rng.normal(size=T)).astype(np.float64) if with_ref else None
    mask = np.array([1, 0, 1, 1, 0, 2], np.uint8) if masked else None
    kw = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.1, ent_coef=ent, scale=0.25)
    c32 = {k: float(np.float32(v)) for k, v in kw.items()}
    want = O.policy_loss(z, labels, old, adv, ref, mask, **c32)
    logp, loss, kl, entropy = (torch.full((T,), 9.0, device=DEV) for _ in range(4))
    d, d_whole = strided(torch.full((T, V), 5.0, dtype=zd.dtype, device=DEV), extra)
    dm = None if mask is None else torch.from_numpy(mask).to(DEV)
    B.bk_policy_loss(zd, lab, f32(old), f32(adv), logp, loss, d, mask=dm, ref_logp=None if ref is None else f32(ref), kl_tok=kl,
                     entropy=entropy, **kw)
    b, rel = logp_bounds(z)
    p = np.exp(O.log_softmax(z))
    lp = O.log_softmax(z)
    within(logp, want[0], b, "logp")
    r = np.exp(now - old)
    grow = np.exp(ref - now) if ref is not None else 0.0
    b_ent = b + (p * (np.abs(lp) + 1) * rel).sum(1) + E * 200 * (p * np.abs(lp)).sum(1)
    b_kl = (b + 4 * E) * np.abs(grow - 1) + 4 * E * (grow + np.abs(now) + 1) * (ref is not None)
    b_c = np.abs(r * adv) * (b + 8 * E * (1 + np.abs(now))) + c32["kl_coef"] * (b_kl + grow * (b + 4 * E)) + 8 * E
    within(entropy, want[3], b_ent, "entropy")
    within(kl, want[2], b_kl, "kl")
    within(loss, want[1], b_c + c32["kl_coef"] * b_kl + ent * b_ent + 8 * E * np.abs(want[1]), "loss")
    c = np.abs(r * adv) + c32["kl_coef"] * np.abs(grow - 1)
    hit = np.zeros(z.shape)
    hit[np.arange(T), labels] = 1
    b_d = b_c[:, None] * (hit + p) + p * (rel + 8 * E) * (c[:, None] + ent * (np.abs(lp) + want[3][:, None])) + \
        ent * p * (b[:, None] + b_ent[:, None]) + hit * 4 * E * c[:, None]
    within(d, want[4], c32["scale"] * b_d + unit(dtype) * np.abs(want[4]) + 1e-38, "dlogits")
    if mask is not None:
        assert not host(d)[mask == 0].any()
    if extra:
        assert bool((d_whole[:, V:] == 7).all())
    # without the gradient, and with the gradient in the logits' place: the same bits
    more = [torch.empty_like(t) for t in (logp, loss)]
    B.bk_policy_loss(zd, lab, f32(old), f32(adv), *more, mask=dm, ref_logp=None if ref is None else f32(ref), **kw)
    assert torch.equal(more[0], logp) and torch.equal(more[1], loss)
    B.bk_policy_loss(zd, lab, f32(old), f32(adv), logp, loss, zd, mask=dm, ref_logp=None if ref is None else f32(ref), kl_tok=kl,
                     entropy=entropy, **kw)
    assert torch.equal(zd, d)


@pytest.mark.parametrize("V", [300, 140001])
def test_policy_loss_of_logits_that_are_not_finite(B, V):
    """-inf takes no part (the type's lowest value neither), rows that count nothing are not read, a NaN stays in its row"""
    T = 6
    z, zd, labels, lab, now = loss_inputs(np.random.default_rng(1), T, V, 1, 0)
    labels[:] = 3
    lab.fill_(3)
    z[0, 10:200] = -np.inf
    z[1, 10:200] = -3.3e38
    z[2, 7] = np.nan
    z[3, 7] = np.nan
    z[4, :] = -np.inf
    zd.copy_(torch.from_numpy(z).to(DEV))
    mask = torch.tensor([1, 1, 1, 0, 1, 1], dtype=torch.uint8, device=DEV)
    one = torch.ones(T, device=DEV)
    out = [torch.empty(T, device=DEV) for _ in range(3)]
    d = torch.empty(T, V, dtype=torch.bfloat16, device=DEV)
    B.bk_policy_loss(zd, lab, -one, one, out[0], out[1], d, mask=mask, entropy=out[2], ent_coef=0.1)
    rows = [0, 1, 5]
    want = O.policy_loss(np.maximum(z[rows], -1e30), labels[rows], -np.ones(3), np.ones(3), ent_coef=0.1)
    for got, w in zip(out[:2] + [out[2]], (want[0], want[1], want[3])):
        assert np.allclose(host(got)[rows], w, rtol=0, atol=200 * E * 20)
    assert np.all(np.abs(host(d)[rows] - want[4]) <= unit(1) * np.abs(want[4]) + 1e-5)
    assert not host(d)[:2, 10:200].any() and not host(d)[3].any()
    assert all(float(t[3]) == 0.0 for t in out)
    assert all(bool(t[i].isnan()) for t in out for i in (2, 4)) and bool(d[2].isnan().all()) and bool(d[4].isnan().all())


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("pairs,seq,V,extra,smoothing", [(1, 1, 7, 0, 0.0), (3, 5, 2051, 2, 0.1), (2, 300, 100, 0, 0.0),
                                                         (1, 3, 50257, 0, 0.25), (1, 2, 140001, 1, 0.0)])
def test_preference_loss(B, dtype, pairs, seq, V, extra, smoothing):
    rng = np.random.default_rng(V + seq)
    n, T = 2 * pairs, 2 * pairs * seq
    z, zd, labels, lab, now = loss_inputs(rng, T, V, dtype, extra)
    mask = (rng.random(T) < 0.7).astype(np.uint8) if seq > 1 else None
    if mask is not None:
        mask[:seq] = 0                                   # a sequence of which nothing counts
    counts = np.ones(T) if mask is None else mask
    ref = np.float32((now * counts).reshape(n, seq).sum(1) + rng.normal(size=n)).astype(np.float64)
    beta, sm, scale = (float(np.float32(t)) for t in (0.3, smoothing, 0.5))
    want = O.preference_loss(z, labels, ref, pairs, beta, sm, mask, scale)
    lse, logp = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    seqs, margin, loss = torch.empty(n, device=DEV), torch.empty(pairs, device=DEV), torch.empty(pairs, device=DEV)
    d, d_whole = strided(torch.full((T, V), 5.0, dtype=zd.dtype, device=DEV), extra)
    dm = None if mask is None else torch.from_numpy(mask).to(DEV)
    B.bk_preference_loss_fwd(zd, lab, f32(ref), lse, logp, seqs, margin, loss, beta, smoothing, mask=dm)
    B.bk_preference_loss_bwd(zd, lab, lse, margin, d, beta, smoothing, scale, mask=dm)
    b, rel = logp_bounds(z)
    b_seq = (b * counts).reshape(n, seq).sum(1)
    within(logp, now * counts, b, "logp")
    within(seqs, want[0], b_seq + E * np.abs(want[0]), "sums")
    b_m = beta * (b_seq[:pairs] + b_seq[pairs:]) + E * np.abs(want[1])
    within(margin, want[1], b_m, "margin")
    within(loss, want[2], b_m + 2 * E * np.abs(want[2]), "loss")
    p = np.exp(O.log_softmax(z))
    hit = np.zeros(z.shape)
    hit[np.arange(T), labels] = 1
    g = np.abs(np.tile(1 / (1 + np.exp(-want[1])) - (1 - sm), 2)).repeat(seq)[:, None] * beta * scale
    slip = (np.tile(b_m, 2) / 4).repeat(seq)[:, None] * beta * scale                  # a sigmoid's slope is at most 1/4
    lse_off = E * np.abs(host(lse))[:, None] * 2
    b_d = (slip + 4 * E * g) * (hit + p) + g * p * (rel + lse_off)
    within(d, want[3], b_d + unit(dtype) * np.abs(want[3]) + 1e-38, "dlogits")
    if extra:
        assert bool((d_whole[:, V:] == 7).all())
    B.bk_preference_loss_bwd(zd, lab, lse, margin, zd, beta, smoothing, scale, mask=dm)       # in place
    assert torch.equal(zd, d)


# ---- AdamW ----------------------------------------------------------------------------------------

HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


def adamw_inputs(rng, sizes, offset):
    """tensors cut out of flat buffers, `offset` elements of their own type beyond an aligned start"""
    def cut(dtype, n):
        return torch.zeros(n + offset, dtype=dtype, device=DEV)[offset:]
    gs = [rng.normal(size=n).astype(np.float32) * np.exp(rng.normal(size=n)).astype(np.float32) * 1e-2 for n in sizes]
    ws = [rng.normal(size=n).astype(np.float32) for n in sizes]
    put = lambda arrays, dtype: [cut(dtype, len(a)).copy_(torch.from_numpy(a)) for a in arrays]
    return gs, ws, put, cut


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("sizes", [[1], [256, 1, 255, 257, 5000], [3, 0, 70001], [17 * i + 1 for i in range(95)]])
def test_adamw_32_bits(B, dtype, offset, sizes):
    rng = np.random.default_rng(len(sizes))
    gs, ws, put, cut = adamw_inputs(rng, sizes, offset)
    act = torch.bfloat16 if dtype == 1 else torch.float32
    ms = [rng.normal(size=n).astype(np.float32) * np.float32(1e-2) for n in sizes]
    vs = [np.float32(rng.random(n) * 1e-4) for n in sizes]
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    g, w, m, v, out = put(gs, torch.float32), put(ws, torch.float32), put(ms, torch.float32), put(vs, torch.float32), [cut(act, n) for n in sizes]
    B.bk_adamw_group(g, w, m, v, out, 3, decay=decay, **HYPER)
    for i in range(len(sizes)):
        a = [t.astype(np.float64) for t in (gs[i], ws[i], ms[i], vs[i])]
        W, M, V = O.adamw(*a, 3, 1e-2, 0.9, 0.99, 1e-8, decay[i])
        # three roundings of the terms of m and v; the step: their roots' and ratios' roundings, each unit of the step's size,
        # and of an m that two terms cancel in
        b_m = 4 * E * (np.abs(0.9 * a[2]) + np.abs(0.1 * a[0]))
        within(m[i], M, b_m + 1e-40, "m")
        within(v[i], V, 5 * E * V + 1e-40, "v")
        size = 1e-2 / (1 - 0.9 ** 3) / (np.sqrt(V / (1 - 0.99 ** 3)) + 1e-8)
        bound = size * (b_m + 12 * E * np.abs(M)) + 3 * E * np.abs(a[1])
        within(w[i], W, bound, "master")
        assert torch.equal(out[i], w[i].to(act))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("sizes", [[1], [256, 255, 257, 5000], [70003, 0, 12]])
def test_adamw_8_bits(B, dtype, offset, sizes):
    """three steps from zero moments; each is compared with the oracle's from the state the kernel left"""
    rng = np.random.default_rng(sum(sizes))
    gs, ws, put, cut = adamw_inputs(rng, sizes, offset)
    act = torch.bfloat16 if dtype == 1 else torch.float32
    g, w, out = put(gs, torch.float32), put(ws, torch.float32), [cut(act, n) for n in sizes]
    m, v = ([cut(torch.uint8, n) for n in sizes] for _ in range(2))
    sm, sv = ([cut(torch.float32, -(-n // 256)) for n in sizes] for _ in range(2))
    off = total = 0
    for step in (1, 2, 3):
        before = [[t.cpu().numpy() for t in ts] for ts in (m, v, sm, sv, w)]
        for i, t in enumerate(g):
            gs[i] = rng.normal(size=sizes[i]).astype(np.float32) * np.float32(0.01)
            t.copy_(torch.from_numpy(gs[i]))
        B.bk_adamw_group(g, w, m, v, out, step, decay=0.1, m_scales=sm, v_scales=sv, seed=5, **HYPER)
        for i, n in enumerate(sizes):
            rep = lambda s: np.repeat(s.astype(np.float64), 256)[:n]
            M0 = O.e4m3(before[0][i]) * rep(before[2][i])
            V0 = (O.e4m3(before[1][i]) * rep(before[3][i])) ** 2
            a, W0 = gs[i].astype(np.float64), before[4][i].astype(np.float64)
            W, M, V = O.adamw(a, W0, M0, V0, step, 1e-2, 0.9, 0.99, 1e-8, 0.1)
            size = 1e-2 / (1 - 0.9 ** step) / (np.sqrt(V / (1 - 0.99 ** step)) + 1e-8)
            b_m = 6 * E * (np.abs(0.9 * M0) + np.abs(0.1 * a))
            within(w[i], W, size * (b_m + 14 * E * np.abs(M)) + 3 * E * np.abs(W0), "master")
            assert torch.equal(out[i], w[i].to(act))
            um, uv = O.rounding_bits(n, 5, step, i)
            for codes, scales, x, up, positive in ((m[i], sm[i], M, um, False), (v[i], sv[i], np.sqrt(V), uv, True)):
                if n == 0:
                    continue
                q, s = O.quantise(x, up, positive)
                within(scales, s, 10 * E * s + 1e-40, "scale")
                got = O.e4m3(codes.cpu().numpy())
                # the same code, except where 32 bits end on the other side of the rounding's border: then the next one
                differ = got != q
                near = np.abs(x) / rep(s)
                assert np.all(np.abs(got - q)[differ] <= 2 * O.code_step(near)[differ]), "codes"
                off, total = off + int(differ.sum()), total + n
    # a value within 8 roundings of the border, which lies at most 16 steps up: 8 * 16 * 2^-24 of the values, and a few
    assert off <= 3 + 10 * total * 8 * 16 * E, (off, total)


def test_adamw_8_bits_keeps_small_moments(B):
    """moments that move by less than half a code a step follow their gradients on average"""
    n, steps = 4096, 400
    g = [torch.full((n,), 1e-3, device=DEV)]
    w, out = [torch.zeros(n, device=DEV)], [torch.zeros(n, device=DEV)]
    m, v = [torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV)], [torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV)]
    sm, sv = [torch.zeros(16, device=DEV)], [torch.zeros(16, device=DEV)]
    g[0][::256] = 1.0                                    # sets each block's scale, far above the others
    for step in range(1, steps + 1):
        B.bk_adamw_group(g, w, m, v, out, step, lr=0.0, m_scales=sm, v_scales=sv, seed=11)
    small = torch.ones(n, dtype=torch.bool, device=DEV)
    small[::256] = False
    mean_m = float((m[0].float() * sm[0].repeat_interleave(256))[small].mean())
    root = (v[0].float() * sv[0].repeat_interleave(256))[small]
    assert abs(mean_m - 1e-3) < 5e-5                     # a mean of 4080 with a step of at most an eighth: 1e-3 / 8 / 64 = 2e-6
    assert float(root.min()) > 0.0
    want = math.sqrt((1 - 0.999 ** steps) * 1e-6)
    # the root is what is rounded: its mean lags by up to its variance, a step of an eighth squared over twice the root
    assert abs(float(root.mean()) - want) < 0.1 * want


def test_adamw_gradients_that_are_not_finite_stay_in_their_place(B):
    for bits in (32, 8):
        n = 1024
        g = torch.ones(n, device=DEV)
        g[300] = float("nan")
        w, out = torch.ones(n, device=DEV), torch.ones(n, device=DEV)
        if bits == 32:
            state, scales = [torch.zeros(n, device=DEV) for _ in range(2)], (None, None)
        else:
            state = [torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2)]
            scales = ([torch.zeros(4, device=DEV)], [torch.zeros(4, device=DEV)])
        for step in (1, 2):
            B.bk_adamw_group([g], [w], [state[0]], [state[1]], [out], step, m_scales=scales[0], v_scales=scales[1])
            g[300] = 1.0
        bad = w.isnan().nonzero().flatten().tolist()
        assert bad == [300], bad


# ---- rows far apart, two calls at once --------------------------------------------------------------------

def test_rows_more_than_32_bits_apart(B):
    """views of one buffer of 6.6 GB: offsets pass 2^32 bytes and 2^31 elements"""
    wide = 1_100_000_000
    buf = torch.empty(3, wide, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(0)
    z, zd = draw(rng, (3, 1000), 1, 2.0)
    buf[:, :1000] = zd
    labels = np.array([1, 999, 500])
    lab = torch.from_numpy(labels.astype(np.int32)).to(DEV)
    one, logp, loss = torch.ones(3, device=DEV), torch.empty(3, device=DEV), torch.empty(3, device=DEV)
    B.bk_policy_loss(buf[:, :1000], lab, -one, one, logp, loss, buf[:, 2000:3000])
    want = O.policy_loss(z, labels, -np.ones(3), np.ones(3))
    assert np.all(np.abs(host(buf[:, 2000:3000]) - want[4]) <= unit(1) * np.abs(want[4]) + 1e-5)
    freq, _ = B.bk_rotary_frequencies(64)
    x, xd = draw(rng, (3, 128), 1)
    buf[:, 4000:4128] = xd
    B.bk_rotary(buf[:, 4000:4128], freq, buf[:, 5000:5128], 2, 64, seq=3)
    turned = O.rotary(x, O.rotary_frequencies(64)[0], np.arange(3), 2, 64)
    within(buf[:, 5000:5128], turned, unit(1) * np.abs(turned) + 1e-5, "rotary")
    # the same memory as 60000 keys of one head, 110 KB apart
    rows = buf.view(-1)[:60000 * 55000].view(60000, 55000)
    rows[:, :128] = torch.randn(60000, 128, device=DEV).bfloat16()
    k, v = rows[:, :64], rows[:, 64:128]
    q, g = torch.randn(4, 64, device=DEV).bfloat16(), torch.randn(4, 64, device=DEV).bfloat16()
    ctx, dq, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(1, 1, 4, device=DEV)
    dk, dv = torch.empty(60000, 64, dtype=torch.bfloat16, device=DEV), torch.empty(60000, 64, dtype=torch.bfloat16, device=DEV)
    B.bk_cross_attention_fwd(q, k, v, ctx, lse, 1, 1)
    B.bk_cross_attention_bwd(q, k, v, ctx, lse, g, dq, dk, dv, 1, 1)
    a = [host(t) for t in (q, k, v, g)]
    want_ctx, want_lse = O.cross_attention_fwd(*a[:3], 1, 1, 1)
    grads = O.cross_attention_bwd(*a, 1, 1, 1)
    bounds = attention_bounds(*a, want_ctx, want_lse, 1, 1, 1, None, unit(1), unit(1))
    for got, w, b in zip((ctx, lse, dq, dk, dv), (want_ctx, want_lse) + grads, bounds):
        within(got, w, b + unit(1) * np.abs(w), "far")


def test_calls_at_once_on_two_streams(B):
    """each call has scratch of its own: two that overlap give what each gives alone"""
    cases = [run_inputs(k) for k in (1, 2)]

    def run(c, stream=None):
        q, k, v, g, n = c
        ctx, dq, dk, dv, lse = (torch.empty_like(t) for t in (q, q, k, v, torch.empty(4, 4, 1, device=DEV)))
        B.bk_cross_attention_fwd(q, k, v, ctx, lse, 4, 4, 2, kv_len=n, stream=stream)
        B.bk_cross_attention_bwd(q, k, v, ctx, lse, g, dq, dk, dv, 4, 4, 2, kv_len=n, stream=stream)
        return ctx, lse, dq, dk, dv
    alone = [run(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        got = [run(c, s) for c, s in zip(cases, streams)]
        torch.cuda.synchronize()
        for x, y in zip(alone, got):
            assert all(torch.equal(a, b) for a, b in zip(x, y))


def run_inputs(seed):
    rng = np.random.default_rng(seed)
    mk = lambda *s: draw(rng, s, 1)[1]
    return mk(4, 256), mk(4 * 3000, 128), mk(4 * 3000, 128), mk(4, 256), torch.tensor([3000, 0, 1, 2999], dtype=torch.int32, device=DEV)


# ---- graphs, streams, one step of them all --------------------------------------------------------------

def test_captured_and_replayed(B):
    """one graph of every operator, replayed with new inputs in its buffers and eager calls of the same kind in between"""
    rng = np.random.default_rng(0)
    batch, sq, sk, heads, d, V = 2, 2, 1200, 4, 64, 5003
    T = batch * sq
    mk = lambda *s: torch.randn(*s, device=DEV).bfloat16()
    freq, _ = B.bk_rotary_frequencies(d)
    q, kv, g, z = mk(T, heads * d), mk(batch * sk, 2 * heads * d), mk(T, heads * d), mk(T, V)
    w = [torch.randn(n, device=DEV) for n in (300, 5)]
    lab = torch.randint(0, V, (T,), dtype=torch.int32, device=DEV)
    old, adv = torch.full((T,), -9.0, device=DEV), torch.randn(T, device=DEV)

    def once(bufs):
        x, ctx, lse, dq, dkv, dz, logp, loss, gs, ms, vs, outs, master = bufs
        H = heads * d
        B.bk_rotary(q, freq, x, heads, d, seq=sq)
        B.bk_cross_attention_fwd(x, kv[:, :H], kv[:, H:], ctx, lse, batch, heads)
        B.bk_cross_attention_bwd(x, kv[:, :H], kv[:, H:], ctx, lse, g, dq, dkv[:, :H], dkv[:, H:], batch, heads)
        B.bk_policy_loss(z, lab, old, adv, logp, loss, dz)
        for m, s in zip(master, w):
            m.copy_(s)
        B.bk_adamw_group(gs, master, ms, vs, outs, 1)
        return [x, ctx, lse, dq, dkv, dz, logp, loss] + master

    def bufs():
        e = torch.empty_like
        return (e(q), e(q), torch.empty(batch, heads, sq, device=DEV), e(q), e(kv), e(z), torch.empty(T, device=DEV),
                torch.empty(T, device=DEV), [torch.ones_like(t) for t in w], [torch.zeros_like(t) for t in w],
                [torch.zeros_like(t) for t in w], [e(t) for t in w], [e(t) for t in w])
    held = bufs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once(bufs())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = once(held)
    for _ in range(3):
        for t in (q, kv, g, z):
            t.copy_(mk(*t.shape))
        for k in (9, 10):
            for t in held[k]:
                t.zero_()
        want = [t.clone() for t in once(bufs())]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(result, want):
            assert torch.equal(a, b)


def test_one_training_step_of_a_decoder_that_reads_an_encoder(B):
    """projection, rotary positions in place, causal attention, attention over encoder states, head, policy loss, the way
    back, AdamW: gradients and new weights against an autograd of the same formulas in 64 bits"""
    torch.manual_seed(0)
    batch, S, sk, heads, kv_heads, d, V = 2, 24, 40, 4, 2, 32, 301
    H, T, Hkv = heads * d, batch * S, kv_heads * d
    shapes = {"Wqkv": (H, 3 * H), "Wq": (H, H), "Wkv": (H, 2 * Hkv), "Wo": (H, V)}
    W = {k: torch.randn(*s, device=DEV) * H ** -0.5 for k, s in shapes.items()}
    x, enc = torch.randn(T, H, device=DEV), torch.randn(batch * sk, H, device=DEV)
    n = torch.tensor([sk, 17], dtype=torch.int32, device=DEV)
    lab = torch.randint(0, V, (T,), dtype=torch.int32, device=DEV)
    adv, old, ref = torch.randn(T, device=DEV), torch.full((T,), -6.0, device=DEV), torch.full((T,), -6.1, device=DEV)
    mask = (torch.rand(T, device=DEV) < 0.7).to(torch.uint8)
    freq, amp = B.bk_rotary_frequencies(d, scaling="linear", factor=2.0)
    new = lambda *s: torch.empty(*s, device=DEV)
    zero = lambda n_: torch.zeros(n_, device=DEV)
    # forward
    qkv, c1, l1 = new(T, 3 * H), new(T, H), new(batch, heads, S)
    B.bk_linear_fwd(x, W["Wqkv"], zero(3 * H), qkv)
    B.bk_rotary(qkv, freq, qkv, 2 * heads, d, seq=S, amplitude=amp)
    B.bk_attention_fwd(qkv, c1, l1, batch, S, heads, True)
    q, kv, c2, l2, z = new(T, H), new(batch * sk, 2 * Hkv), new(T, H), new(batch, heads, S), new(T, V)
    B.bk_linear_fwd(c1, W["Wq"], zero(H), q)
    B.bk_linear_fwd(enc, W["Wkv"], zero(2 * Hkv), kv)
    B.bk_cross_attention_fwd(q, kv[:, :Hkv], kv[:, Hkv:], c2, l2, batch, heads, kv_heads, kv_len=n)
    B.bk_linear_fwd(c2, W["Wo"], zero(V), z)
    # loss and the way back
    logp, loss, dz, total = new(T), new(T), new(T, V), new(1)
    scale = 1.0 / float(mask.sum())
    B.bk_policy_loss(z, lab, old, adv, logp, loss, dz, mask=mask, ref_logp=ref, kl_coef=0.1, ent_coef=0.01, scale=scale)
    B.bk_ordered_sum(loss, scale, total)
    G = {k: torch.zeros(*s, device=DEV) for k, s in shapes.items()}
    dc2, dq, dkv, dc1, dqkv = new(T, H), new(T, H), new(batch * sk, 2 * Hkv), new(T, H), new(T, 3 * H)
    B.bk_linear_bwd_input(dz, W["Wo"], dc2)
    B.bk_linear_bwd_weight(c2, dz, G["Wo"])
    B.bk_cross_attention_bwd(q, kv[:, :Hkv], kv[:, Hkv:], c2, l2, dc2, dq, dkv[:, :Hkv], dkv[:, Hkv:], batch, heads, kv_heads, kv_len=n)
    B.bk_linear_bwd_weight(enc, dkv, G["Wkv"])
    B.bk_linear_bwd_input(dq, W["Wq"], dc1)
    B.bk_linear_bwd_weight(c1, dq, G["Wq"])
    B.bk_attention_bwd(qkv, c1, l1, dc1, dqkv, batch, S, heads, True)
    B.bk_rotary(dqkv, freq, dqkv, 2 * heads, d, seq=S, amplitude=amp, inverse=True)
    B.bk_linear_bwd_weight(x, dqkv, G["Wqkv"])
    # the same in 64 bits
    P = {k: t.double().cpu().requires_grad_(True) for k, t in W.items()}
    f, cpu = O.rotary_frequencies(d, scaling="linear", factor=2.0)[0], lambda t: t.double().cpu()
    ang = (torch.arange(T) % S).double()[:, None, None] * torch.from_numpy(f)
    a = (cpu(x) @ P["Wqkv"]).view(T, 3, heads, d)

    def turned(t):
        u, v = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([u * ang.cos() - v * ang.sin(), v * ang.cos() + u * ang.sin()], -1)

    def attend(q_, k_, v_, mask_):
        s = q_ @ k_.transpose(-1, -2) / math.sqrt(d)
        return torch.softmax(s.masked_fill(~mask_, -math.inf), -1) @ v_
    split = lambda t, h: t.reshape(batch, -1, h, d).transpose(1, 2)
    h1 = attend(split(turned(a[:, 0]), heads), split(turned(a[:, 1]), heads), split(a[:, 2], heads), torch.ones(S, S).tril().bool())
    h1 = h1.transpose(1, 2).reshape(T, H)
    kv64 = (cpu(enc) @ P["Wkv"]).view(batch * sk, 2, kv_heads, d)
    keys = split(kv64[:, 0], kv_heads).repeat_interleave(heads // kv_heads, 1), split(kv64[:, 1], kv_heads).repeat_interleave(heads // kv_heads, 1)
    h2 = attend(split(h1 @ P["Wq"], heads), *keys, (torch.arange(sk) < n.cpu()[:, None])[:, None, None, :].bool())
    lp = torch.log_softmax(h2.transpose(1, 2).reshape(T, H) @ P["Wo"], 1)
    lt = lp.gather(1, lab.cpu().long()[:, None])[:, 0]
    r, A, u = torch.exp(lt - cpu(old)), cpu(adv), cpu(ref) - lt
    per = -torch.minimum(r * A, r.clamp(0.8, 1.2) * A) + 0.1 * (torch.exp(u) - u - 1) + 0.01 * (lp.exp() * lp).sum(1)
    value = (per * (cpu(mask) != 0)).sum() * scale
    grads = torch.autograd.grad(value, list(P.values()))
    # each product and softmax rounds to 32 bits: a chain of eight with sums of up to 301 terms, a thousandth of the storage bar
    value = float(value.detach())
    assert abs(float(total) - value) <= 1e-5 * (abs(value) + 1)
    for (name, want), got in zip(zip(P, grads), G.values()):
        assert float((cpu(got) - want).norm() / want.norm()) <= 1e-4, name
    # and the step, with and without decay, moments in 8 bits for half of the matrices
    names = list(shapes)
    before = {k: W[k].clone() for k in names}
    masters, outs = [W[k].view(-1) for k in names], [torch.empty_like(W[k]).view(-1) for k in names]
    decay = [0.1, 0.0]
    for part in (0, 2):
        ms, vs = ([torch.zeros(t.numel(), dtype=torch.uint8 if part else torch.float32, device=DEV) for t in masters[part:part + 2]]
                  for _ in range(2))
        sc = [[zero(-(-t.numel() // 256)) for t in ms] for _ in range(2)] if part else (None, None)
        B.bk_adamw_group([G[k].view(-1) for k in names[part:part + 2]], masters[part:part + 2], ms, vs, outs[part:part + 2], 1, lr=1e-2,
                         eps=1e-4, decay=decay, m_scales=sc[0], v_scales=sc[1])
    for i, k in enumerate(names):
        w0, g0 = host(before[k]).ravel(), host(G[k]).ravel()
        want = O.adamw(g0, w0, 0 * g0, 0 * g0, 1, 1e-2, 0.9, 0.999, 1e-4, decay[i % 2])[0]
        within(masters[i], want, 20 * E * (np.abs(w0) + 1e-2), k)
