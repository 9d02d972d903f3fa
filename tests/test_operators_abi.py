"""What the operators' entry points refuse, and their host side (no GPU: a call that got past its checks would try a launch
and come back with another status than the one asked for)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2204_12013_amd import binding as B

P, ODD = 1 << 20, (1 << 20) + 1          # addresses that nothing is read from here
P2, P3, P4, P5, P6, P7, P8 = (P + (k << 20) for k in range(1, 8))


@pytest.mark.parametrize("scaling", B.ROTARY_SCALINGS)
@pytest.mark.parametrize("rot,base,factor,length", [(2, 10000.0, 4.0, 128), (64, 500000.0, 8.0, 4096), (50, 1000.0, 1.0, 77)])
def test_rotary_frequencies(scaling, rot, base, factor, length):
    freq, amp = B.bk_rotary_frequencies(rot, base, scaling, factor, length, device="cpu")
    want, want_amp = O.rotary_frequencies(rot, base, scaling, factor, length)
    # pow in 64 bits on both sides, each within 1 unit; the amplitude is handed over in 32 bits
    assert freq.dtype == torch.float64 and np.allclose(freq.numpy(), want, rtol=8 * 2.0 ** -52, atol=0)
    assert abs(amp - want_amp) <= 2.0 ** -24 * want_amp


@pytest.mark.parametrize("args", [
    (3, 10.0, "none", 1.0, 0), (0, 10.0, "none", 1.0, 0), (4, 1.0, "none", 1.0, 0), (4, float("nan"), "none", 1.0, 0),
    (4, 10.0, "linear", 0.5, 0), (4, 10.0, "stretched", float("inf"), 0), (4, 10.0, "parts", 2.0, 0), (4, 10.0, "other", 1.0, 0)])
def test_rotary_frequencies_refuses(args):
    with pytest.raises(B.BambooError) as e:
        B.bk_rotary_frequencies(*args, device="cpu")
    assert e.value.status == B.E_ARG


ROTARY = dict(dtype=1, T=4, seq=4, heads=2, d=64, rot=64, interleaved=0, inverse=0, x=P, ldx=128, pos=None, freq=P, amp=1.0, y=P,
              ldy=128, stream=None)
CROSS = dict(dtype=1, impl=0, batch=2, sq=3, sk=5, heads=4, kv_heads=2, d=64, q=P, ldq=256, k=P2, v=P3, ldkv=128, kv_len=None, ctx=P4,
             ldc=256, lse=P, scratch=P, stream=None)
CROSS_BWD = dict(dtype=1, impl=0, batch=2, sq=3, sk=5, heads=4, kv_heads=2, d=64, q=P, ldq=256, k=P2, v=P3, ldkv=128, kv_len=None,
                 ctx=P4, ldc=256, lse=P, dctx=P5, lddc=256, dq=P6, lddq=256, dk=P7, dv=P8, lddkv=128, scratch=P, stream=None)
POLICY = dict(dtype=1, T=4, V=100, logits=P, ldl=100, labels=P, mask=None, old=P, ref=None, adv=P, clip_low=0.2, clip_high=0.2,
              kl=0.0, ent=0.0, scale=1.0, logp=P, loss=P, kl_tok=None, entropy=None, dlogits=P, ldd=100, stream=None)
PREF = dict(dtype=1, pairs=2, seq=3, V=100, logits=P, ldl=100, labels=P, mask=None, ref=P, beta=0.1, smoothing=0.0, lse=P, logp=P,
            logp_seq=P, margin=P, loss=P, scratch=P, stream=None)
PREF_BWD = dict(dtype=1, pairs=2, seq=3, V=100, logits=P, ldl=100, labels=P, mask=None, lse=P, margin=P, beta=0.1, smoothing=0.0,
                scale=1.0, dlogits=P, ldd=100, stream=None)


@pytest.mark.parametrize("name,good,bad", [
    ("bk_rotary", ROTARY, [dict(dtype=2), dict(T=0), dict(heads=0), dict(rot=63), dict(rot=66), dict(rot=0), dict(d=1, rot=2), dict(d=514),
                           dict(ldx=127), dict(ldy=127), dict(x=None), dict(y=None), dict(freq=None), dict(seq=0), dict(x=ODD),
                           dict(y=P + 2), dict(y=P + 256), dict(ldy=130), dict(y=P - 128 * 2)]),
    ("bk_cross_attention_fwd", CROSS, [dict(dtype=-1), dict(impl=3), dict(batch=0), dict(sq=0), dict(sk=0), dict(heads=3), dict(kv_heads=0),
                                       dict(d=129), dict(d=0), dict(ldq=255), dict(ldkv=127), dict(ldc=255), dict(q=None), dict(k=None),
                                       dict(v=None), dict(ctx=None), dict(lse=None), dict(q=ODD), dict(scratch=P + 4),
                                       dict(sq=1 << 30, heads=8, ldq=512, ldc=512), dict(batch=1 << 30), dict(ctx=P), dict(ctx=P2 + 128),
                                       dict(ctx=P3)]),
    ("bk_cross_attention_bwd", CROSS_BWD, [dict(scratch=None), dict(dctx=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(lddc=255),
                                           dict(lddq=255), dict(lddkv=127), dict(dk=ODD), dict(heads=5), dict(dq=P), dict(dq=P5), dict(dk=P2),
                                           dict(dv=P3 + 64), dict(dv=P7), dict(dk=P6), dict(dq=P4)]),
    ("bk_policy_loss", POLICY, [dict(dtype=3), dict(T=0), dict(V=0), dict(ldl=99), dict(ldd=99), dict(logits=None), dict(labels=None),
                                dict(old=None), dict(adv=None), dict(logp=None), dict(loss=None), dict(logits=ODD), dict(clip_low=-0.1),
                                dict(clip_low=1.5), dict(clip_high=float("nan")), dict(dlogits=P + 2), dict(ldd=101),
                                dict(V=(1 << 27) + 1, ldl=1 << 28, ldd=1 << 28)]),
    ("bk_preference_loss_fwd", PREF, [dict(dtype=3), dict(pairs=0), dict(seq=0), dict(V=0), dict(ldl=99), dict(logits=None), dict(labels=None),
                                      dict(ref=None), dict(lse=None), dict(logp=None), dict(logp_seq=None), dict(margin=None),
                                      dict(loss=None), dict(smoothing=1.5), dict(pairs=1 << 20, seq=1 << 12), dict(scratch=None),
                                      dict(scratch=P + 4)]),
    ("bk_preference_loss_bwd", PREF_BWD, [dict(lse=None), dict(margin=None), dict(dlogits=None), dict(ldd=99), dict(dlogits=P + 4),
                                          dict(ldd=102), dict(smoothing=-0.1)]),
])
def test_refused_arguments(name, good, bad):
    for change in bad:
        assert getattr(B.lib, name)(*dict(good, **change).values()) == B.E_ARG, (name, change)


@pytest.mark.parametrize("name,change", [
    ("bk_rotary", dict(ldx=300, ldy=300, y=P + 2 * 128)),               # queries beside the rotated ones, in one matrix
    ("bk_rotary", dict(ldx=300, ldy=300, y=P + 2 * 172)),
    ("bk_policy_loss", dict(ldl=200, ldd=200, dlogits=P + 2 * 100)),
    ("bk_cross_attention_bwd", dict(ldkv=256, v=P2 + 2 * 128, lddkv=256, dv=P7 + 2 * 128))])
def test_columns_beside_each_other_are_not_refused(name, change):
    good = {"bk_rotary": ROTARY, "bk_policy_loss": POLICY, "bk_cross_attention_bwd": CROSS_BWD}[name]
    if torch.cuda.is_available():
        pytest.skip("the addresses are none: without a GPU the launch itself is what fails")
    assert getattr(B.lib, name)(*dict(good, **change).values()) == B.E_HIP


def test_forced_bf16_attention_does_not_take_fp32():
    assert B.lib.bk_cross_attention_fwd(*dict(CROSS, impl=2, dtype=0).values()) == B.E_STATE
    assert B.lib.bk_cross_attention_bwd(*dict(CROSS_BWD, impl=2, dtype=0).values()) == B.E_STATE


def _adamw(n=2, dtype=1, bits=32, numel=(8, 8), g=(P, P), master=(P, P + 4096), m=(P, P), v=(P, P), ms=None, vs=None, w=(P, P),
           decay=(0.0, 0.0), b1=0.9, b2=0.999, eps=1e-8, step=1):
    ptrs = lambda t: None if t is None else (C.c_void_p * len(t))(*t)
    return B.lib.bk_adamw_group(dtype, bits, n, (C.c_int64 * 2)(*numel), ptrs(g), ptrs(master), ptrs(m), ptrs(v), ptrs(ms), ptrs(vs),
                                ptrs(w), (C.c_double * 2)(*decay), 1e-3, b1, b2, eps, step, 0, None)


@pytest.mark.parametrize("change", [
    dict(n=0), dict(dtype=2), dict(bits=16), dict(step=0), dict(numel=(8, -1)), dict(g=(P, None)), dict(master=None), dict(w=(P, ODD)),
    dict(m=(P, P + 2)), dict(master=(P, P)), dict(master=(P, P + 16)), dict(b1=1.0), dict(b2=-0.1), dict(eps=float("nan")),
    dict(bits=8), dict(bits=8, ms=(P, P)), dict(bits=8, ms=(P, None), vs=(P, P)), dict(ms=(P, P), vs=(P, P))])
def test_adamw_refuses(change):
    assert _adamw(**change) == B.E_ARG


def test_adamw_of_nothing_launches_nothing():
    assert _adamw(numel=(0, 0), g=(None, None), master=(None, None)) == B.OK


def test_scratch_is_asked_for_where_parts_are_joined():
    f = B.lib.bk_cross_attention_scratch_floats
    assert f(8, 512, 64, 64, 64, 64) == 8 * 64 * 512                        # delta of the backward alone
    assert f(1, 1, 8192, 8, 8, 64) > 8 * 64
    assert f(0, 1, 1, 1, 1, 1) == 0 and f(1, 1, 1, 3, 2, 1) == 0


def test_tensors_that_do_not_fit_are_refused():
    bf, f32 = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, 128)
    freq = torch.zeros(32, dtype=torch.float64)
    vec = lambda n, t=torch.float32: torch.zeros(n, dtype=t)
    lab = vec(4, torch.int32)
    for call in [
        lambda: B.bk_rotary(bf, freq, f32, 2, 64),                                        # two dtypes
        lambda: B.bk_rotary(bf.half(), freq, bf.half(), 2, 64),                           # one that there is not
        lambda: B.bk_rotary(bf.t(), freq, bf.t(), 1, 4),                                  # columns apart
        lambda: B.bk_rotary(bf, freq, bf, 3, 64),                                         # more heads than columns
        lambda: B.bk_cross_attention_fwd(bf, bf, bf[:2], bf, vec(8), 2, 2),               # fewer values than keys
        lambda: B.bk_cross_attention_fwd(bf, bf, f32, bf, vec(8), 2, 2),
        lambda: B.bk_cross_attention_fwd(bf, bf, bf, bf, vec(8), 3, 2),                   # rows are not whole samples
        lambda: B.bk_cross_attention_fwd(bf, bf[:, :64], torch.zeros(4, 256, dtype=torch.bfloat16)[:, :64], bf, vec(8), 2, 2, 1),
        lambda: B.bk_policy_loss(bf, lab, vec(4), vec(4), vec(4), vec(4), f32),           # a gradient of another dtype
        lambda: B.bk_policy_loss(bf, lab, vec(4), vec(4), vec(4), vec(4), bf[:3]),
        lambda: B.bk_preference_loss_fwd(bf, lab, vec(6), vec(4), vec(4), vec(6), vec(3), vec(3), 0.1),
        lambda: B.bk_preference_loss_bwd(bf, lab, vec(4), vec(3), bf, 0.1),
        lambda: B.bk_adamw_group([f32], [f32], [f32], [f32], [bf, bf], 1),
        lambda: B.bk_adamw_group([f32], [f32], [f32], [f32[:2]], [bf], 1),
        lambda: B.bk_adamw_group([bf], [f32], [f32], [f32], [bf], 1),
        lambda: B.bk_adamw_group([f32], [f32], [f32], [f32], [bf], 1, decay=[0.1, 0.1]),
        lambda: B.bk_adamw_group([f32], [f32], [vec(512, torch.uint8)], [vec(512, torch.uint8)], [bf], 1, m_scales=[vec(3)],
                                 v_scales=[vec(2)]),
        lambda: B.bk_adamw_group([], [], [], [], [], 1),
    ]:
        with pytest.raises(B.BambooError) as e:
            call()
        assert e.value.status == B.E_ARG
