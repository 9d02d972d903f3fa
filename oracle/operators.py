"""Operators around the stage, in plain numpy float64, one function per formula (no blocking, no fusion).

rotary positions, softmax attention over states of another length with shared key heads and key lengths, a clipped policy
loss and a preference loss on the log-probability of given tokens with their gradients, AdamW with moments in 32 or in 8 bits.
"""
import math

import numpy as np


# ---- rotary positions ---------------------------------------------------------------------------

def rotary_frequencies(rot, base=10000.0, scaling="none", factor=1.0, length=0):
    """(angle per position of each pair, factor on the turned vectors)"""
    if scaling == "stretched" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "parts":
        kept = np.clip((length * f / (2 * math.pi) - 1) / 31, 0, 1)
        return f * (kept + (1 - kept) / factor), 0.1 * math.log(factor) + 1
    return f, 1.0


def rotary(x, freq, pos, heads, d, interleaved=False, inverse=False, amplitude=1.0):
    """x [T, heads*d]; the first 2 len(freq) features of every head turned by pos * freq."""
    y, n = x.reshape(len(x), heads, d).copy(), len(freq)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    angle = np.asarray(pos, np.float64)[:, None, None] * freq
    c, s = np.cos(angle) * amplitude, np.sin(-angle if inverse else angle) * amplitude
    u, v = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return y.reshape(x.shape)


# ---- attention over an encoder's states ---------------------------------------------------------

def _heads(q, k, v, batch, heads, kv_heads, kv_len):
    """(sample, head, rows of q, rows of k, columns of q, columns of k) of each softmax"""
    sq, sk, d = len(q) // batch, len(k) // batch, q.shape[1] // heads
    for b in range(batch):
        n = sk if kv_len is None else min(max(int(kv_len[b]), 0), sk)
        for h in range(heads):
            kh = h // (heads // kv_heads)
            yield b, h, slice(b * sq, (b + 1) * sq), slice(b * sk, b * sk + n), slice(h * d, h * d + d), slice(kh * d, kh * d + d)


def cross_attention_fwd(q, k, v, batch, heads, kv_heads, kv_len=None):
    ctx, lse = np.zeros(q.shape), np.full((batch, heads, len(q) // batch), -np.inf)
    for b, h, rq, rk, cq, ck in _heads(q, k, v, batch, heads, kv_heads, kv_len):
        if rk.start == rk.stop:
            continue
        z = q[rq, cq] @ k[rk, ck].T / math.sqrt(q.shape[1] // heads)
        top = z.max(1, keepdims=True)
        e = np.exp(z - top)
        total = e.sum(1, keepdims=True)
        ctx[rq, cq] = e / total @ v[rk, ck]
        lse[b, h] = (top + np.log(total))[:, 0]
    return ctx, lse


def cross_attention_bwd(q, k, v, dctx, batch, heads, kv_heads, kv_len=None):
    ctx, lse = cross_attention_fwd(q, k, v, batch, heads, kv_heads, kv_len)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    scale = 1 / math.sqrt(q.shape[1] // heads)
    for b, h, rq, rk, cq, ck in _heads(q, k, v, batch, heads, kv_heads, kv_len):
        if rk.start == rk.stop:
            continue
        p = np.exp(q[rq, cq] @ k[rk, ck].T * scale - lse[b, h][:, None])
        g = dctx[rq, cq]
        ds = p * (g @ v[rk, ck].T - (g * ctx[rq, cq]).sum(1, keepdims=True)) * scale
        dq[rq, cq] = ds @ k[rk, ck]
        dk[rk, ck] += ds.T @ q[rq, cq]
        dv[rk, ck] += p.T @ g
    return dq, dk, dv


# ---- losses on given tokens ---------------------------------------------------------------------

def log_softmax(z):
    top = z.max(1, keepdims=True)
    return z - top - np.log(np.exp(z - top).sum(1, keepdims=True))


def policy_loss(z, labels, old, adv, ref=None, mask=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, ent_coef=0.0, scale=1.0):
    """logp, loss, kl, entropy per token, and scale times the gradient at the logits"""
    lp = log_softmax(z)
    p, T = np.exp(lp), len(z)
    with np.errstate(invalid="ignore"):
        plogp = np.where(p > 0, p * lp, 0.0)
    logp, entropy = lp[np.arange(T), labels], -plogp.sum(1)
    r = np.exp(logp - old)
    free, held = r * adv, np.clip(r, 1 - clip_low, 1 + clip_high) * adv
    loss, c, kl = -np.minimum(free, held) - ent_coef * entropy, np.where(free <= held, -free, 0.0), np.zeros(T)
    if ref is not None:
        u = ref - logp
        kl = np.expm1(u) - u
        loss, c = loss + kl_coef * kl, c - kl_coef * np.expm1(u)
    hit = np.zeros(z.shape)
    hit[np.arange(T), labels] = 1
    d = c[:, None] * (hit - p) + ent_coef * (plogp + p * entropy[:, None])
    counts = np.ones(T) if mask is None else (np.asarray(mask) != 0) * 1.0
    keep = lambda t: np.where(counts > 0, t, 0.0)
    return keep(logp), keep(loss), keep(kl), keep(entropy), np.where(counts[:, None] > 0, d * scale, 0.0)


def preference_loss(z, labels, ref, pairs, beta, smoothing=0.0, mask=None, scale=1.0):
    """sums of log-probabilities, margin and loss per pair, and scale times the gradient of the losses at the logits"""
    lp, T = log_softmax(z), len(z)
    counts = np.ones(T) if mask is None else (np.asarray(mask) != 0) * 1.0
    seqs = np.where(counts > 0, lp[np.arange(T), labels], 0.0).reshape(2 * pairs, -1).sum(1)
    margin = beta * ((seqs - ref)[:pairs] - (seqs - ref)[pairs:])
    loss = (1 - smoothing) * np.logaddexp(0, -margin) + smoothing * np.logaddexp(0, margin)
    g = beta * (1 / (1 + np.exp(-margin)) - (1 - smoothing))
    c = np.repeat(np.concatenate([g, -g]), T // (2 * pairs)) * counts
    hit = np.zeros(z.shape)
    hit[np.arange(T), labels] = 1
    return seqs, margin, loss, np.where(counts[:, None] > 0, scale * c[:, None] * (hit - np.exp(lp)), 0.0)


# ---- AdamW --------------------------------------------------------------------------------------

def adamw(g, master, m, v, step, lr, beta1, beta2, eps, decay):
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    w = master * (1 - lr * decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w, m, v


def e4m3(codes):
    """values of one-byte codes: sign, 4 bits of exponent (bias 7), 3 of the fraction; no infinities"""
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    mag = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c >> 7, -mag, mag)


def _mix(x):
    """an integer hash of 32 bits (C. Wellons, "Prospecting for Hash Functions", 2018)"""
    m = np.uint64(0xFFFFFFFF)
    x = np.asarray(x, np.uint64)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x7FEB352D)) & m
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x846CA68B)) & m
    return x ^ (x >> np.uint64(16))


def rounding_bits(n, seed, step, tensor):
    """two numbers in (0, 1) for each of n elements: which way the first and the root of the second moment are rounded"""
    key = _mix((int(_mix((seed + step * 0x9E3779B9) & 0xFFFFFFFF)) + tensor * 0x85EBCA6B) & 0xFFFFFFFF)
    h = _mix(np.arange(n, dtype=np.uint64) ^ key)
    return ((h & np.uint64(0xFFFF)).astype(np.float64) + 0.5) / 65536, ((h >> np.uint64(16)).astype(np.float64) + 0.5) / 65536


def code_step(q):
    """distance between the codes around q >= 0"""
    _, e = np.frexp(q)
    return 2.0 ** (np.maximum(e - 1, -6) - 3)


def quantise(x, up, positive):
    """(values in units of the scale, scale per block of 256): rounded down, or up where the part beyond it and `up` make a step"""
    blocks = -(-len(x) // 256)
    top = np.abs(np.pad(x, (0, blocks * 256 - len(x)))).reshape(blocks, 256).max(1)
    inv = np.where(top > 1e-30, 448 / np.where(top > 0, top, 1), 0)
    q = np.minimum(np.abs(x) * np.repeat(inv, 256)[:len(x)], 448.0)
    s = code_step(q)
    n = np.minimum(np.floor(q / s + up) * s, 448.0)
    if positive:
        n = np.where(x > 0, np.maximum(n, 2.0 ** -9), n)
    return np.sign(x) * n, top / 448
