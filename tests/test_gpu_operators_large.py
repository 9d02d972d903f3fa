"""Operators around the stage in the forms that large batches run (GPU only): every number of threads and vectors a row of the
policy loss, results that bypass the caches (calls that move more than 384 MB), against the 64-bit oracle on chosen rows and ranges."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from test_gpu_operators import B, DEV, E, f32, host, unit, within  # noqa: F401  (B is a fixture)
from test_gpu_operators_edges import check_policy, row_bounds, stored

pytestmark = pytest.mark.gpu
FORMS = [(256, 1), (256, 2), (256, 4), (256, 6), (256, 8), (256, 12), (256, 16), (512, 10), (512, 13), (512, 16), (1024, 12), (1024, 16)]


def plain(V, n=3):
    rng = np.random.default_rng(V)
    return rng.standard_normal((n, V)) * 2.5, rng.integers(0, V, n)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("threads,vectors", FORMS)
def test_policy_loss_of_every_row_length(B, dtype, threads, vectors):
    """rows that fill a form to its last vector, and one that ends inside it"""
    V = threads * vectors * (8 if dtype == 1 else 4)
    check_policy(B, *plain(V), dtype, T=300)
    check_policy(B, *plain(V - 3), dtype, T=300, extra=5)


@pytest.mark.parametrize("dtype,T,V,extra", [(1, 4100, 50304, 0), (1, 4100, 50257, 3), (0, 4100, 32003, 0), (1, 2050, 140001, 1), (0, 600, 90000, 0)])
@pytest.mark.parametrize("ent", [0.01, 0.0])
def test_policy_loss_past_the_caches(B, dtype, T, V, extra, ent):
    assert 2 * T * V * (2 if dtype == 1 else 4) > 384 << 20
    check_policy(B, *plain(V), dtype, T=T, extra=extra, ent=ent, with_ref=False)


@pytest.mark.parametrize("dtype,pairs,seq,V,extra", [(1, 4, 520, 50257, 1), (1, 8, 300, 50304, 0), (0, 3, 700, 32003, 2), (1, 2, 200, 9001, 0)])
def test_preference_loss_of_many_rows(B, dtype, pairs, seq, V, extra):
    """three tokens of a sequence count, those and a few others are looked at; the last shape stays within the caches"""
    rng = np.random.default_rng(V)
    n, T, act = 2 * pairs, 2 * pairs * seq, torch.bfloat16 if dtype == 1 else torch.float32
    rows = np.sort(np.concatenate([i * seq + rng.permutation(seq)[:3] for i in range(n)]))
    at = torch.from_numpy(rows).to(DEV)
    z, labels = plain(V, len(rows))
    z = stored(z, dtype)
    logits = torch.full((T, V + extra), float("nan"), dtype=act, device=DEV)[:, :V]
    logits[at] = torch.from_numpy(z).to(DEV).to(act)
    lab = torch.zeros(T, dtype=torch.int32, device=DEV)
    lab[at] = torch.from_numpy(labels.astype(np.int32)).to(DEV)
    mask = torch.zeros(T, dtype=torch.bool, device=DEV)
    mask[at] = True
    lp, b, rel = row_bounds(z, labels)
    now = lp[np.arange(len(rows)), labels]
    beta, sm, scale = 0.25, 0.125, 0.5                                  # held exactly
    ref = np.float32(now.reshape(n, 3).sum(1) + rng.normal(size=n)).astype(np.float64)
    want = O.preference_loss(z, labels, ref, pairs, beta, sm, None, scale)
    lse, logp, seqs = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(n, device=DEV)
    margin, loss = torch.empty(pairs, device=DEV), torch.empty(pairs, device=DEV)
    whole = torch.full((T, V + extra), 5.0, dtype=act, device=DEV)
    d = whole[:, :V]
    B.bk_preference_loss_fwd(logits, lab, f32(ref), lse, logp, seqs, margin, loss, beta, sm, mask=mask)
    B.bk_preference_loss_bwd(logits, lab, lse, margin, d, beta, sm, scale, mask=mask)
    b_seq = b.reshape(n, 3).sum(1)
    b_m = beta * (b_seq[:pairs] + b_seq[pairs:]) + E * np.abs(want[1])
    within(logp[at], now, b, "logp")
    within(seqs, want[0], b_seq + E * np.abs(want[0]), "sums")
    within(margin, want[1], b_m, "margin")
    within(loss, want[2], b_m + 2 * E * np.abs(want[2]), "loss")
    hit = np.zeros(z.shape)
    hit[np.arange(len(rows)), labels] = 1
    p = np.exp(lp)
    g = np.abs(np.tile(1 / (1 + np.exp(-want[1])) - (1 - sm), 2)).repeat(3)[:, None] * beta * scale
    slip = (np.tile(b_m, 2) / 4).repeat(3)[:, None] * beta * scale         # a sigmoid's slope is at most 1/4
    b_d = (slip + 4 * E * g) * (hit + p) + g * p * (rel + E * np.abs(host(lse[at]))[:, None] * 2)
    within(d[at], want[3], b_d + unit(dtype) * np.abs(want[3]) + 1e-38, "dlogits")
    left = ~mask
    assert not bool(d[left].any()) and not bool(logp[left].any()) and (not extra or bool((whole[:, V:] == 5).all()))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_adamw_past_the_caches(B, dtype, bits, offset):
    """24 M parameters, one tensor almost all of them: its two ends and its middle, and the small ones beside it"""
    sizes = [257, 24_000_001, 3]
    rng = np.random.default_rng(bits + offset)
    act, hyper = torch.bfloat16 if dtype == 1 else torch.float32, dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)
    cut = lambda t, n: torch.zeros(n + offset, dtype=t, device=DEV)[offset:]
    fill = lambda n, by: cut(torch.float32, n).normal_().mul_(by)
    torch.manual_seed(bits)
    g, w, out = [fill(n, 0.01) for n in sizes], [fill(n, 1.0) for n in sizes], [cut(act, n) for n in sizes]
    mt = torch.float32 if bits == 32 else torch.uint8
    m, v = ([cut(mt, n) for n in sizes] for _ in range(2))
    sm, sv = ([cut(torch.float32, -(-n // 256)) for n in sizes] for _ in range(2)) if bits == 8 else (None, None)
    off = total = 0
    for step in (1, 2):                                                     # each compared from the state that the kernel left
        ranges = [(i, a, min(a + 4096, n)) for i, n in enumerate(sizes) for a in sorted({0, n // 512 * 256, max(0, n // 256 * 256 - 2048)})]
        take = lambda ts: [ts[i][a:e].cpu().numpy() for i, a, e in ranges]
        blocks = lambda ts: [ts[i][a // 256:-(-e // 256)].cpu().numpy().astype(np.float64) for i, a, e in ranges]
        before = [take(t) for t in (g, w, m, v)] + ([blocks(sm), blocks(sv)] if bits == 8 else [])
        B.bk_adamw_group(g, w, m, v, out, step, decay=0.1, m_scales=sm, v_scales=sv, seed=9, **hyper)
        after = [take(t) for t in (w, m, v)] + ([blocks(sm), blocks(sv)] if bits == 8 else [])
        noise = {i: O.rounding_bits(n, 9, step, i) for i, n in enumerate(sizes)} if bits == 8 else None
        for k, (i, a, e) in enumerate(ranges):
            G, W0 = before[0][k].astype(np.float64), before[1][k].astype(np.float64)
            rep = lambda s: np.repeat(s, 256)[:e - a]
            if bits == 32:
                M0, V0 = before[2][k].astype(np.float64), before[3][k].astype(np.float64)
            else:
                M0, V0 = O.e4m3(before[2][k]) * rep(before[4][k]), (O.e4m3(before[3][k]) * rep(before[5][k])) ** 2
            W, M, V = O.adamw(G, W0, M0, V0, step, 1e-2, 0.9, 0.99, 1e-8, 0.1)
            b_m = 6 * E * (np.abs(0.9 * M0) + np.abs(0.1 * G))
            size = 1e-2 / (1 - 0.9 ** step) / (np.sqrt(V / (1 - 0.99 ** step)) + 1e-8)
            within(after[0][k].astype(np.float64), W, size * (b_m + 14 * E * np.abs(M)) + 3 * E * np.abs(W0), "master")
            if bits == 32:
                within(after[1][k].astype(np.float64), M, b_m + 1e-40, "m")
                within(after[2][k].astype(np.float64), V, 5 * E * V + 1e-40, "v")
                continue
            for codes, scales, x, up, positive in ((after[1][k], after[3][k], M, noise[i][0], False), (after[2][k], after[4][k], np.sqrt(V), noise[i][1], True)):
                q, s = O.quantise(x, up[a:e], positive)
                within(scales, s, 10 * E * s + 1e-40, "scale")
                got = O.e4m3(codes)
                differ, near = got != q, np.abs(x) / rep(s)
                assert np.all(np.abs(got - q)[differ] <= 2 * O.code_step(near)[differ]), "codes"
                off, total = off + int(differ.sum()), total + e - a
        assert all(torch.equal(o, t.to(act)) for o, t in zip(out, w))
    assert off <= 3 + 10 * total * 8 * 16 * E, (off, total)                 # near a border of the rounding, as in the small tests
