"""Sizes and factors at the ends of the ranges that the policy update's headers give: refused with the documented code, before anything is enqueued."""
import pytest

from paper_2512_21450_amd import binding as B
from test_abi_policy_update import attn, attn_grad


@pytest.mark.parametrize("kw", [dict(T=1 << 24, Hq=1 << 12, Hkv=1 << 12, d=64), dict(T=1 << 23, Hq=3 << 11, Hkv=1 << 11, d=128)])
def test_packed_attn_grids_beyond_2_32_threads(kw):
    """blocks of rows or keys times their threads: HIP runs a launch of 2^32 threads and more in part"""
    q, k = dict(q_stride=kw["Hq"] * kw["d"]), dict(k_stride=kw["Hkv"] * kw["d"], v_stride=kw["Hkv"] * kw["d"])
    assert B.rl_packed_attn_raw(attn(**kw, **q, **k, out_stride=q["q_stride"])) == -2
    grads = dict(dout_stride=q["q_stride"], dq_stride=q["q_stride"], dk_stride=k["k_stride"], dv_stride=k["k_stride"])
    assert B.rl_packed_attn_backward_raw(attn_grad(**kw, **q, **k, out_stride=q["q_stride"], **grads, workspace=0x1000, workspace_bytes=1 << 60)) == -2


def test_packed_attn_backward_grid_of_key_blocks():
    """64 heads of one key each: blocks of keys have more threads than blocks of rows"""
    kw = dict(T=1 << 21, Hq=256, Hkv=256, d=64, q_stride=256 * 64, k_stride=256 * 64, v_stride=256 * 64, out_stride=256 * 64)
    grads = dict(dout_stride=256 * 64, dq_stride=256 * 64, dk_stride=256 * 64, dv_stride=256 * 64, workspace=0x1000, workspace_bytes=1 << 60)
    assert B.rl_packed_attn_backward_raw(attn_grad(**kw, **grads)) == -2


@pytest.mark.parametrize("scale", [2.5e38, -3e38])
def test_scales_whose_base_2_form_is_no_number(scale):
    assert B.rl_packed_attn_raw(attn(scale=scale)) == -1 and B.rl_packed_attn_backward_raw(attn_grad(scale=scale)) == -1
    assert B.rl_packed_attn_backward_workspace_bytes(attn_grad(scale=scale)) == 0


@pytest.mark.parametrize("T,S,Hq,Hkv,d,parts", [(3136, 1, 8, 8, 64, 1), (3136, 3, 16, 8, 128, 1), (6272, 1, 4, 4, 128, 1), (8448, 1, 2, 2, 128, 2), (4000, 1, 28, 4, 128, 2),
                                                (6272, 16, 28, 4, 128, 2), (1100, 1, 28, 4, 128, 3), (7040, 1, 28, 4, 128, 1)])
def test_packed_attn_workgroups_that_share_a_block_of_keys(T, S, Hq, Hkv, d, parts):
    """only where their sums, which the workspace holds, are worth writing: one sequence of few rows for so many blocks gains nothing by it"""
    plain = T * Hq * 8 + (T + 63) // 64 * 8
    need = B.rl_packed_attn_backward_workspace_bytes(B.make_packed_attn_backward_desc(T, S, Hq, Hkv, d, 0.1))
    assert need == plain if parts == 1 else need == (plain + 255) // 256 * 256 + parts * 2 * T * Hkv * d * 4
