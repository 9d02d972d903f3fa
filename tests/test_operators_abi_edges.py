"""More of what the operators' entry points take and refuse, on the host (no GPU: a call that got past its checks would try a launch
and come back with another status than the one asked for)."""
import pytest
import torch

from paper_2204_12013_amd import binding as B
from test_operators_abi import CROSS, CROSS_BWD, P, P2, POLICY, PREF, PREF_BWD, ROTARY, _adamw


def test_the_row_distance_of_a_single_row_says_nothing():
    """one token through views of different widths: in place, and into columns beside each other"""
    row, columns = dict(ROTARY, T=1, pos=P), dict(CROSS_BWD, batch=1, sq=1, sk=1, ldkv=256, v=P2 + 2 * 128)
    assert B.lib.bk_rotary(*dict(row, y=P + 2, ldy=300).values()) == B.E_ARG
    assert B.lib.bk_cross_attention_bwd(*dict(columns, dk=P2 + 2 * 64).values()) == B.E_ARG
    assert B.lib.bk_cross_attention_bwd(*dict(columns, dq=P2 + 2 * 200, lddq=1000).values()) == B.E_ARG
    if torch.cuda.is_available():
        pytest.skip("the addresses are none: without a GPU the launch itself is what fails")
    for change in (dict(ldx=300), dict(ldy=300), dict(ldx=128, ldy=1 << 33), dict(y=P + 2 * 128, ldy=300)):
        assert B.lib.bk_rotary(*dict(row, **change).values()) == B.E_HIP
    assert B.lib.bk_policy_loss(*dict(POLICY, T=1, ldd=200).values()) == B.E_HIP


MOST = (1 << 24) - 1          # workgroups of 256 threads in a launch


@pytest.mark.parametrize("name,good,bad,last", [
    ("bk_policy_loss", POLICY, dict(T=MOST + 1), dict(T=MOST)),
    ("bk_preference_loss_fwd", PREF, dict(pairs=MOST // 2 + 1, seq=1), dict(pairs=MOST // 2, seq=1)),
    ("bk_preference_loss_bwd", PREF_BWD, dict(pairs=1, seq=MOST // 2 + 1), dict(pairs=1, seq=MOST // 2))])
def test_more_rows_than_a_launch_has_workgroups_are_refused(name, good, bad, last):
    assert getattr(B.lib, name)(*dict(good, **bad).values()) == B.E_ARG
    if not torch.cuda.is_available():      # the addresses are none: without a GPU the launch itself is what fails
        assert getattr(B.lib, name)(*dict(good, **last).values()) == B.E_HIP


def test_more_elements_than_a_launch_can_take_are_refused():
    assert _adamw(numel=(8, MOST * 1024 + 1), master=(P, P + 4096)) == B.E_ARG
    if not torch.cuda.is_available():
        assert _adamw(numel=(8, MOST * 1024), master=(P, P + 4096)) == B.E_HIP


@pytest.mark.parametrize("sizes", [(1, 1 << 30, 4, 1 << 30, 1, 128), (1 << 20, 1 << 20, 1 << 20, 8, 8, 64), (1 << 30, 1, 1, 4, 4, 64),
                                   (1, 1 << 16, 1, 1 << 16, 1, 1), (1, 1, 0x7FFFFFFF, 1, 1, 1)])
def test_no_scratch_for_sizes_that_are_refused(sizes):
    """their products pass 64 bits, or what a launch can have"""
    batch, sq, sk, heads, kv_heads, d = sizes
    assert B.lib.bk_cross_attention_scratch_floats(*sizes) == 0
    big = dict(batch=batch, sq=sq, sk=sk, heads=heads, kv_heads=kv_heads, d=d, ldq=heads * d, ldkv=kv_heads * d, ldc=heads * d)
    assert B.lib.bk_cross_attention_fwd(*dict(CROSS, **big).values()) == B.E_ARG
