"""Operators around the stage where their inputs are unusual, and in the forms that large batches run (GPU only), against the
64-bit oracle with derived bounds.  Units as in test_gpu_operators: u half a step of the storage type, E that of fp32."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2204_12013_amd import synth
from test_gpu_operators import B, DEV, E, f32, host, unit, within  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


# ---- losses ---------------------------------------------------------------------------------------

def stored(z, dtype):
    """the values that the storage type holds, as float64"""
    return synth.round_to_storage(np.asarray(z, np.float32), dtype).astype(np.float64)


def row_bounds(z, labels):
    """(log-probabilities, error of a label's, relative error of a probability, per row and element)"""
    at = np.arange(len(z))
    t = z.max(1, keepdims=True) - z
    lp = O.log_softmax(z)
    p = np.exp(lp)
    t0 = np.where(p > 0, t, 0.0)
    # exponents: two roundings of t log2 e each; sums of at most 128 terms a thread (V / 1024 of longer rows), then 22 more.  The
    # maximum itself cancels: logits enter as differences to it, and what its own product is rounded by is taken back
    s = E * (4 * (p * t0).sum(1) + max(128, z.shape[1] / 512) + 30)
    b = s + E * (8 + t[at, labels] + 2 * np.abs(np.log(np.exp(-t).sum(1))))
    return lp, b, E * 4 * (t0 + 2) + b[:, None]


def check_policy(B, z, labels, dtype, T=None, extra=0, ent=0.01, with_ref=True, scale=0.25):
    """the rows of z among T rows of which no other counts: all outputs"""
    n, V = z.shape
    T = n if T is None else T
    rng = np.random.default_rng(V)
    z = stored(z, dtype)
    rows = np.sort(rng.permutation(T)[:n])
    act = torch.bfloat16 if dtype == 1 else torch.float32
    logits = torch.full((T, V + extra), float("nan"), dtype=act, device=DEV)[:, :V]
    logits[torch.from_numpy(rows).to(DEV)] = torch.from_numpy(z).to(DEV).to(act)
    lp, b, rel = row_bounds(z, labels)
    p, at = np.exp(lp), np.arange(n)
    now = lp[at, labels]
    old, ref = (np.float32(now + k * rng.normal(size=n)).astype(np.float64) for k in (0.2, 0.4))
    adv = np.float32(rng.normal(size=n)).astype(np.float64)
    kw = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.1, ent_coef=ent, scale=scale)
    c32 = {k: float(np.float32(v)) for k, v in kw.items()}
    want = O.policy_loss(z, labels, old, adv, ref if with_ref else None, None, **c32)

    def spread(x, dtype=torch.float32):
        t = torch.full((T,), 3, dtype=dtype, device=DEV)
        t[torch.from_numpy(rows).to(DEV)] = torch.from_numpy(np.asarray(x)).to(DEV).to(dtype)
        return t
    mask = torch.zeros(T, dtype=torch.uint8, device=DEV)
    mask[torch.from_numpy(rows).to(DEV)] = 1
    logp, loss, kl, entropy = (torch.full((T,), 9.0, device=DEV) for _ in range(4))
    whole = torch.full((T, V + extra), 5.0, dtype=act, device=DEV)
    d = whole[:, :V]
    args = (spread(labels, torch.int32), spread(old), spread(adv), logp, loss)
    keep = dict(mask=mask, ref_logp=spread(ref) if with_ref else None, kl_tok=kl, entropy=entropy, **kw)
    B.bk_policy_loss(logits, *args, d, **keep)
    lp0 = np.where(p > 0, lp, 0.0)
    r = np.exp(now - old)
    grow = np.exp(ref - now) if with_ref else 0.0
    b_ent = b + (p * (np.abs(lp0) + 1) * rel).sum(1) + E * 200 * (p * np.abs(lp0)).sum(1)
    b_kl = (b + 4 * E) * np.abs(grow - 1) + 4 * E * (grow + np.abs(now) + 1) * with_ref
    b_c = np.abs(r * adv) * (b + 8 * E * (1 + np.abs(now))) + c32["kl_coef"] * (b_kl + grow * (b + 4 * E)) + 8 * E
    got = lambda t: host(t)[rows]
    within(got(logp), want[0], b, "logp")
    within(got(entropy), want[3], b_ent, "entropy")
    within(got(kl), want[2], b_kl, "kl")
    within(got(loss), want[1], b_c + c32["kl_coef"] * b_kl + ent * b_ent + 8 * E * np.abs(want[1]), "loss")
    c = np.abs(r * adv) + c32["kl_coef"] * np.abs(grow - 1)
    hit = np.zeros(z.shape)
    hit[at, labels] = 1
    b_d = b_c[:, None] * (hit + p) + p * (rel + 8 * E) * (c[:, None] + ent * (np.abs(lp0) + want[3][:, None])) + \
        ent * p * (b[:, None] + b_ent[:, None]) + hit * 4 * E * c[:, None]
    chosen = d[torch.from_numpy(rows).to(DEV)]
    within(chosen, want[4], c32["scale"] * b_d + unit(dtype) * np.abs(want[4]) + 1e-38, "dlogits")
    left = torch.ones(T, dtype=torch.bool, device=DEV)
    left[torch.from_numpy(rows).to(DEV)] = False
    assert not bool(d[left].any()) and all(not bool(t[left].any()) for t in (logp, loss, kl, entropy))
    assert not extra or bool((whole[:, V:] == 5).all())
    B.bk_policy_loss(logits, *args, logits, **keep)                             # in place: the same bits
    assert torch.equal(logits, d)


def banned(V, values):
    """six rows of logits with a share of them at `values`, and labels that may be chosen: one row's own is a low one"""
    rng = np.random.default_rng(V)
    z, labels = rng.standard_normal((6, V)) * 2.5, rng.integers(V // 2, V, 6)
    for row in range(5):
        z[row, :V // 2] = np.where(rng.random(V // 2) < 0.3, values[row % len(values)], z[row, :V // 2])
    z[5, labels[5]] = -95.0
    z[0, V - 1], labels[0] = values[0], V - 2
    return z, labels


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [6, 300])
@pytest.mark.parametrize("V", [100, 300, 4096, 32000, 50304, 140001])
@pytest.mark.parametrize("ent", [0.01, 0.0])
def test_policy_loss_of_tokens_that_are_all_but_ruled_out(B, dtype, T, V, ent):
    """logits so far below the row's maximum that their probability is 0 in 32 bits: all outputs finite and right"""
    check_policy(B, *banned(V, [-95.0, -100.0, -1e4, -1e9, -1e30]), dtype, T=T, ent=ent)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V", [100, 300, 2051, 4096, 32003, 50257, 140001])
def test_policy_loss_of_tokens_that_are_ruled_out(B, dtype, V):
    """logits of -inf take no part, in vocabularies that fill their last vector and that do not"""
    check_policy(B, *banned(V, [-np.inf]), dtype)


def level(V, dtype):
    """six rows whose largest logits are far from 0, several of them alike, and labels among those"""
    low = float(torch.finfo(torch.bfloat16 if dtype == 1 else torch.float32).min)
    rng = np.random.default_rng(V)
    z = np.tile(np.array([low, -1e30, -1e10, -3e6, 1e30, -2e30])[:, None], (1, V))
    z[3] += rng.integers(0, 2, V) * (1 << 16)                          # two levels, both held exactly
    z[4, :V // 2] = 0.0
    z[5, V // 3:] = low
    z[1, :V // 4] = -np.inf
    return z, np.array([V - 1, V - 1, 0, int(z[3].argmax()), V - 1, 0])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [6, 300])
@pytest.mark.parametrize("V", [100, 2051, 32000, 50304, 140001])
def test_policy_loss_of_rows_far_from_zero(B, dtype, T, V):
    """a row that a mask has set to the type's lowest value, or to another far one, throughout: the tokens are alike"""
    check_policy(B, *level(V, dtype), dtype, T=T)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("pairs,V", [(3, 100), (300, 2051), (3, 140001)])
def test_sequences_of_rows_far_from_zero(B, dtype, pairs, V):
    z, labels = level(V, dtype)
    z, n = stored(z, dtype), 2 * pairs
    pick = np.arange(n) % 6
    act = torch.bfloat16 if dtype == 1 else torch.float32
    zd = torch.from_numpy(z).to(DEV).to(act)[torch.from_numpy(pick).to(DEV)]
    lse, logp, seqs = (torch.empty(n, device=DEV) for _ in range(3))
    margin, loss = torch.empty(pairs, device=DEV), torch.empty(pairs, device=DEV)
    lp, b, _ = row_bounds(z, labels)
    now, b = lp[np.arange(6), labels][pick], b[pick]
    B.bk_preference_loss_fwd(zd, torch.from_numpy(labels[pick].astype(np.int32)).to(DEV), f32(np.zeros(n)), lse, logp, seqs, margin, loss, 0.5)
    within(logp, now, b, "logp")
    within(seqs, now, b, "sums")
    within(margin, 0.5 * (now[:pairs] - now[pairs:]), b[:pairs] + b[pairs:], "margin")


def test_preference_loss_of_a_sequence_that_cannot_be(B):
    """a label of probability 0: the margin is infinite, and a side of the loss that has no weight adds nothing"""
    pairs, V = 3, 50
    z = torch.randn(2 * pairs, V, device=DEV)
    lab = torch.full((2 * pairs,), 7, dtype=torch.int32, device=DEV)
    z[3, 7] = z[1, 7] = -float("inf")                                           # rejected of pair 0, chosen of pair 1
    for smoothing, want in ((0.0, [0.0, np.inf]), (1.0, [np.inf, 0.0]), (0.25, [np.inf, np.inf])):
        lse, logp, seqs = (torch.empty(2 * pairs, device=DEV) for _ in range(3))
        margin, loss, d = torch.empty(pairs, device=DEV), torch.empty(pairs, device=DEV), torch.empty_like(z)
        B.bk_preference_loss_fwd(z, lab, torch.zeros(2 * pairs, device=DEV), lse, logp, seqs, margin, loss, 0.5, smoothing)
        B.bk_preference_loss_bwd(z, lab, lse, margin, d, 0.5, smoothing)
        assert margin[:2].tolist() == [np.inf, -np.inf]
        assert loss[:2].tolist() == want and bool(loss[2].isfinite())
        assert bool(d.isfinite().all())


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_preference_gradient_of_pairs_that_are_told_apart_well(B, dtype, smoothing):
    """margins at which a sigmoid is 1 to the last bit, and the gradient its difference to 1"""
    rng = np.random.default_rng(5)
    margins = np.array([60.0, -60.0, 35.0, -35.0, 18.0, -18.0, 0.25])
    pairs, V = len(margins), 200
    z = stored(rng.normal(size=(2 * pairs, V)), dtype)
    labels = rng.integers(0, V, 2 * pairs)
    zd = torch.from_numpy(z).to(DEV).to(torch.bfloat16 if dtype == 1 else torch.float32)
    lp = O.log_softmax(z)
    lse = f32(z[:, 0] - lp[:, 0])
    d, sm = torch.empty_like(zd), float(np.float32(smoothing))
    B.bk_preference_loss_bwd(zd, torch.from_numpy(labels.astype(np.int32)).to(DEV), lse, f32(margins), d, 0.5, smoothing)
    g = 0.5 * (sm / (1 + np.exp(-margins)) - (1 - sm) / (1 + np.exp(margins)))
    hit = np.zeros(z.shape)
    hit[np.arange(2 * pairs), labels] = 1
    c, p = np.concatenate([g, -g])[:, None], np.exp(lp)
    # the coefficient rounded once, an exponential of a difference to a rounded lse, a product and a difference
    bound = np.abs(c) * (E * hit + p * E * (8 + 4 * np.abs(lp) + 2 * np.abs(host(lse))[:, None]))
    within(d, c * (hit - p), bound + (unit(dtype) + 2 * E) * np.abs(c * (hit - p)) + 1e-38, "dlogits")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V", [100, 2051, 140001])
def test_policy_loss_of_a_label_that_cannot_be(B, dtype, V):
    """its probability is 0 and its KL term infinite, not NaN; without weight the term adds nothing to loss and gradient"""
    T, label = 4, 7
    act = torch.bfloat16 if dtype == 1 else torch.float32
    z = torch.randn(T, V, device=DEV).to(act)
    z[1, label] = z[2, 3] = -float("inf")
    lab, one = torch.full((T,), label, dtype=torch.int32, device=DEV), torch.ones(T, device=DEV)
    for coef in (0.0, 0.1):
        logp, loss, kl, ent = (torch.empty(T, device=DEV) for _ in range(4))
        d = torch.empty_like(z)
        B.bk_policy_loss(z, lab, -one, one, logp, loss, d, ref_logp=-one, kl_tok=kl, entropy=ent, kl_coef=coef, ent_coef=0.1)
        assert float(logp[1]) == -np.inf and float(kl[1]) == np.inf
        fine = torch.tensor([True, coef == 0.0, True, True], device=DEV)
        assert bool(loss[fine].isfinite().all()) and bool(d[fine].isfinite().all()) and bool(ent.isfinite().all())
        assert coef == 0.0 or float(loss[1]) == np.inf


# ---- attention over an encoder's states -------------------------------------------------------------

@pytest.mark.parametrize("garbage", [float("nan"), float("inf")])
@pytest.mark.parametrize("sq,heads,kv_heads,d", [(40, 4, 2, 64), (3000, 1, 1, 128), (9, 6, 2, 33)])
@pytest.mark.parametrize("dtype,impl", [(0, 0), (1, 2), (1, 1)])
def test_rows_that_are_not_finite_stay_among_what_they_meet(B, dtype, impl, sq, heads, kv_heads, d, garbage):
    """a query or a gradient that is not finite: keys that do not count keep their zeros, other rows and samples their values"""
    batch, sk, n = 3, 150, [70, 0, 129]
    act = torch.bfloat16 if dtype == 1 else torch.float32
    mk = lambda rows, cols: torch.randn(rows, cols, device=DEV).to(act)
    q, k, v, g = mk(batch * sq, heads * d), mk(batch * sk, kv_heads * d), mk(batch * sk, kv_heads * d), mk(batch * sq, heads * d)
    lens = torch.tensor(n, dtype=torch.int32, device=DEV)

    def run(q, g):
        ctx, dq, dk, dv, lse = (torch.full_like(t, 3.0) for t in (q, q, k, v, torch.empty(batch, heads, sq, device=DEV)))
        B.bk_cross_attention_fwd(q, k, v, ctx, lse, batch, heads, kv_heads, kv_len=lens, impl=impl)
        B.bk_cross_attention_bwd(q, k, v, ctx, lse, g, dq, dk, dv, batch, heads, kv_heads, kv_len=lens, impl=impl)
        return ctx, dq, dk, dv
    clean = run(q, g)
    for which, sample in (("q", 0), ("g", 2), ("g", 0), ("q", 2)):
        bad_q, bad_g = q.clone(), g.clone()
        row = sample * sq + sq // 2
        (bad_q if which == "q" else bad_g)[row, d // 2] = garbage
        got = run(bad_q, bad_g)
        for b in range(batch):
            for t, c in zip(got[2:], clean[2:]):
                rows = slice(b * sk + n[b], (b + 1) * sk)
                assert not bool(t[rows].any()), (which, b)
                if b != sample:
                    assert torch.equal(t[b * sk:(b + 1) * sk], c[b * sk:(b + 1) * sk]), (which, b)
        others = torch.arange(batch * sq, device=DEV) != row
        for t, c in zip(got[:2], clean[:2]):
            assert torch.equal(t[others], c[others]), which


@pytest.mark.parametrize("sq,heads,kv_heads,d,lens", [(4, 4, 2, 64, [3, 2500, 70, 128, 0]), (1, 8, 2, 128, [1, 3000, 100, 2]), (3, 2, 2, 80, [5, 2000, 127]),
                                                      (130, 2, 2, 64, [3, 128, 65])])
def test_gradients_of_queries_over_few_keys(B, sq, heads, kv_heads, d, lens):
    """Samples of at most 128 keys, beside long ones that have the launch cut into parts and without: dQ has the roundings of dS and of
    itself, none from the rounded context."""
    rng = np.random.default_rng(sum(lens))
    batch, sk, u = len(lens), max(lens), unit(1)
    scale = d ** -0.5
    q, k, v, g = (stored(rng.standard_normal((batch * rows, cols)) * mul, 1) for rows, cols, mul in
                  ((sq, heads * d, 1.3), (sk, kv_heads * d, 1.0), (sk, kv_heads * d, 1.0), (sq, heads * d, 0.1)))
    put = lambda t: torch.from_numpy(t).to(DEV).to(torch.bfloat16)
    qd, kd, vd, gd = put(q), put(k), put(v), put(g)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ctx, dq, dk, dv, lse = torch.empty_like(qd), torch.empty_like(qd), torch.empty_like(kd), torch.empty_like(vd), torch.empty(batch, heads, sq, device=DEV)
    B.bk_cross_attention_fwd(qd, kd, vd, ctx, lse, batch, heads, kv_heads, kv_len=n)
    B.bk_cross_attention_bwd(qd, kd, vd, ctx, lse, gd, dq, dk, dv, batch, heads, kv_heads, kv_len=n)
    want, bound = np.zeros(q.shape), np.zeros(q.shape)
    for b, h, rq, rk, cq, ck in O._heads(q, k, v, batch, heads, kv_heads, lens):
        m = rk.stop - rk.start
        if m == 0 or m > 128:
            bound[rq, cq] = np.inf if m else 0.0
            continue
        z = q[rq, cq] @ k[rk, ck].T * scale
        p = np.exp(O.log_softmax(z))
        gv, mags = g[rq, cq] @ v[rk, ck].T, np.abs(g[rq, cq]) @ np.abs(v[rk, ck]).T
        delta = (p * gv).sum(1, keepdims=True)
        ds = p * (gv - delta)
        want[rq, cq] = scale * ds @ k[rk, ck]
        # a probability: d products and sums of the score, its scale and exponent, the log-sum-exp's own sum of m terms
        rel = E * ((d + 4) * (np.abs(q[rq, cq]) @ np.abs(k[rk, ck]).T) * scale + 8 * np.abs(z).max() + m + 16) * 2
        b_delta = (p * (rel * np.abs(gv) + E * (d + 8) * mags)).sum(1, keepdims=True)
        b_ds = p * (rel * np.abs(gv - delta) + b_delta + E * (d + 8) * (mags + np.abs(delta))) + u * np.abs(ds)
        bound[rq, cq] = scale * (b_ds @ np.abs(k[rk, ck]) * (1 + 4 * u) + E * (m + 8) * (np.abs(ds) @ np.abs(k[rk, ck]))) + u * np.abs(want[rq, cq])
    small = np.isfinite(bound).all(1)
    within(host(dq)[small], want[small], bound[small] + 1e-38, "dq")


# ---- rotary positions -------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [1, 2, 9])
def test_rotary_in_place_through_a_narrower_view(B, dtype, T):
    """queries and keys of a packed row written over themselves, the values beside them kept: one token as well as many"""
    act = torch.bfloat16 if dtype == 1 else torch.float32
    x = torch.randn(T, 3 * 2 * 64, device=DEV).to(act)
    freq, _ = B.bk_rotary_frequencies(64)
    pos = torch.arange(1000, 1000 + T, dtype=torch.int32, device=DEV)
    want = torch.empty(T, 256, dtype=act, device=DEV)
    B.bk_rotary(x, freq, want, 4, 64, pos=pos)
    values = x[:, 256:].clone()
    B.bk_rotary(x, freq, x[:, :256], 4, 64, pos=pos)
    assert torch.equal(x[:, :256], want) and torch.equal(x[:, 256:], values)


# ---- AdamW ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_adamw_8_bits_of_a_gradient_that_is_not_finite(B, bad):
    """NaN in its element's moments, or in its block's where it sets the block's scale; nothing else differs"""
    n, at = 1024, 300

    def run(value, steps):
        torch.manual_seed(3)
        g, w, out = torch.randn(n, device=DEV), torch.randn(n, device=DEV), torch.empty(n, device=DEV)
        m, v = (torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
        sm, sv = torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
        for step in range(1, steps + 1):
            if step == 1 and value is not None:
                g[at] = value
            B.bk_adamw_group([g], [w], [m], [v], [out], step, m_scales=[sm], v_scales=[sv], seed=4)
            g[at] = 1.0
        return m.float() * sm.repeat_interleave(256), v.float() * sv.repeat_interleave(256), w, out
    block = torch.zeros(n, dtype=torch.bool, device=DEV)
    block[256:512] = True
    only = torch.zeros_like(block)
    only[at] = True
    for steps in (1, 2):
        clean, got = run(None, steps), run(bad, steps)
        moments = block if abs(bad) == float("inf") else only
        for i, (c, t) in enumerate(zip(clean, got)):
            broken = moments if i < 2 or steps == 2 else only
            assert bool(t[broken].isnan().all()), (i, steps)
            assert torch.equal(t[~block], c[~block]) and bool(t[~broken].isfinite().all()), (i, steps)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr,decay", [(1e-4, 0.01), (1e-5, 0.1), (3e-5, 0.002), (1e-3, 0.1)])
def test_adamw_decays_weights_to_their_last_bit(B, bits, lr, decay):
    """no gradient and no moments: what is left is w - lr decay w, whose one rounding is the weight's own"""
    n = 1 << 16
    w0 = np.float32(np.random.default_rng(2).normal(size=n))
    w, out, g = f32(w0), torch.empty(n, device=DEV), torch.zeros(n, device=DEV)
    state = [torch.zeros(n, dtype=torch.float32 if bits == 32 else torch.uint8, device=DEV) for _ in range(2)]
    scales = [[torch.zeros(n // 256, device=DEV)] for _ in range(2)] if bits == 8 else (None, None)
    B.bk_adamw_group([g], [w], [state[0]], [state[1]], [out], 1, lr=lr, decay=decay, m_scales=scales[0], v_scales=scales[1])
    a = w0.astype(np.float64)
    # the decayed part has two roundings of its own (of lr decay and of the product), 2 E of it
    within(w, a * (1 - lr * decay), E * np.abs(a) + 3 * E * lr * decay * np.abs(a), "master")


# ---- sizes -------------------------------------------------------------------------------------------

def test_sizes_that_pass_32_bits_are_refused(B):
    """handed over in 32 bits they would be those of four rows"""
    x = torch.empty(2 ** 32 + 4, 2, dtype=torch.bfloat16, device=DEV)
    freq, _ = B.bk_rotary_frequencies(2)
    q, lse = torch.ones(1, 2, dtype=torch.bfloat16, device=DEV), torch.empty(1, device=DEV)
    for call in (lambda: B.bk_rotary(x, freq, x, 1, 2), lambda: B.bk_cross_attention_fwd(q, x, x, q.clone(), lse, 1, 1)):
        with pytest.raises(B.BambooError) as e:
            call()
        assert e.value.status == B.E_ARG


# ---- graphs ------------------------------------------------------------------------------------------

def test_losses_keys_and_8_bit_moments_captured_and_replayed(B):
    """what replays with new inputs in its buffers, key lengths among them, with eager calls of the same kind in between"""
    pairs, seq, V, batch, sk, heads, d, n = 2, 3, 4099, 2, 900, 4, 64, 3000
    T = 2 * pairs * seq
    bf = lambda *s: torch.randn(*s, device=DEV).bfloat16()
    z, z2, q, kv, g = bf(T, V), bf(T, V), bf(batch, heads * d), bf(batch * sk, 2 * heads * d), bf(batch, heads * d)
    lens, grad, ref = torch.tensor([sk, 0], dtype=torch.int32, device=DEV), torch.randn(n, device=DEV), torch.randn(2 * pairs, device=DEV)
    lab, mask = torch.randint(0, V, (T,), dtype=torch.int32, device=DEV), torch.ones(T, dtype=torch.uint8, device=DEV)
    one = torch.ones(T, device=DEV)
    master, codes, scales = torch.randn(n, device=DEV), torch.randint(0, 120, (2, n), dtype=torch.uint8, device=DEV), torch.rand(2, 12, device=DEV)
    f = lambda *s: torch.empty(*s, device=DEV)

    def bufs():
        return dict(lse=f(T), logp=f(T), seqs=f(2 * pairs), margin=f(pairs), loss=f(pairs), d=torch.empty_like(z), d2=torch.empty_like(z),
                    tok=f(T), kl=f(T), ent=f(T), logp2=f(T), ctx=torch.empty_like(q), st=f(batch, heads, 1), dq=torch.empty_like(q),
                    dkv=torch.empty_like(kv), w=f(n), out=f(n), c=torch.empty_like(codes), s=torch.empty_like(scales))

    def once(b):
        H = heads * d
        B.bk_preference_loss_fwd(z, lab, ref, b["lse"], b["logp"], b["seqs"], b["margin"], b["loss"], 0.1, 0.1, mask=mask)
        B.bk_preference_loss_bwd(z, lab, b["lse"], b["margin"], b["d"], 0.1, 0.1, mask=mask)
        B.bk_policy_loss(z2, lab, -one, one, b["logp2"], b["tok"], b["d2"], mask=mask, ref_logp=-one, kl_tok=b["kl"], entropy=b["ent"],
                         kl_coef=0.1, ent_coef=0.1)
        B.bk_cross_attention_fwd(q, kv[:, :H], kv[:, H:], b["ctx"], b["st"], batch, heads, kv_len=lens)
        B.bk_cross_attention_bwd(q, kv[:, :H], kv[:, H:], b["ctx"], b["st"], g, b["dq"], b["dkv"][:, :H], b["dkv"][:, H:], batch, heads,
                                 kv_len=lens)
        for k, t in (("w", master), ("c", codes), ("s", scales)):
            b[k].copy_(t)
        B.bk_adamw_group([grad], [b["w"]], [b["c"][0]], [b["c"][1]], [b["out"]], 7, m_scales=[b["s"][0]], v_scales=[b["s"][1]], seed=3)
        return b
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once(bufs())
    torch.cuda.current_stream().wait_stream(side)
    held, graph = bufs(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once(held)
    for k in range(3):
        for t in (z, z2, q, kv, g, grad, ref, master):
            t.copy_(torch.randn(t.shape, device=DEV))
        lab.random_(0, V)
        mask.random_(0, 2)
        lens.copy_(torch.tensor([[1, sk], [0, 0], [65, 700]][k], dtype=torch.int32))
        want = once(bufs())
        graph.replay()
        torch.cuda.synchronize()
        for name in held:
            a, b = held[name], want[name]
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (k, name)
