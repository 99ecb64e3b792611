"""CPU-side checks of the rotary calls: refusals (before anything is launched) and the positions of a plan's rows."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2605_08524_amd as fcp
from paper_2605_08524_amd import binding as B

OK = dict(head_dim=64, n_pairs=16, n_axes=2, interleaved=0, axis=[0, 1] * 8, turn=[2 ** 60] * 16)
PART = dict(src=4096, dst=8192, pos=4096, src_row_stride=128, dst_row_stride=128, n_rows=3, n_heads=2, src_f32=0, dst_f32=0)


def _call(spec, part, n_parts=1, **null):
    s = dict(OK, **spec)
    axis, turn = np.asarray(s.pop("axis"), dtype=np.int32), np.asarray(s.pop("turn"), dtype=np.uint64)
    r = B._Rotary(axis=None if null.get("axis") else axis.ctypes.data, turn=None if null.get("turn") else turn.ctypes.data, **s)
    parts = (B._RotaryPart * max(1, n_parts))(*[B._RotaryPart(**dict(PART, **part))] * max(1, min(n_parts, 4)))
    return B._lib.fcp_rotary_apply(None if null.get("r") else C.byref(r), None if null.get("parts") else parts, n_parts, 0, None)


@pytest.mark.parametrize("spec,part,code", [
    (dict(head_dim=72), {}, B.FCP_ERR_UNSUPPORTED), (dict(head_dim=0), {}, B.FCP_ERR_UNSUPPORTED), (dict(head_dim=272), {}, B.FCP_ERR_UNSUPPORTED),
    (dict(n_pairs=12), {}, B.FCP_ERR_UNSUPPORTED), (dict(n_pairs=0), {}, B.FCP_ERR_UNSUPPORTED), (dict(n_pairs=40), {}, B.FCP_ERR_UNSUPPORTED),
    (dict(n_axes=0), {}, B.FCP_ERR_INVALID_ARG), (dict(n_axes=9), {}, B.FCP_ERR_INVALID_ARG), (dict(n_axes=1), {}, B.FCP_ERR_INVALID_ARG),
    (dict(axis=[-1] * 16), {}, B.FCP_ERR_INVALID_ARG),
    ({}, dict(src=None), B.FCP_ERR_INVALID_ARG), ({}, dict(dst=None), B.FCP_ERR_INVALID_ARG), ({}, dict(pos=None), B.FCP_ERR_INVALID_ARG),
    ({}, dict(n_rows=-1), B.FCP_ERR_INVALID_ARG), ({}, dict(n_heads=0), B.FCP_ERR_INVALID_ARG),
    ({}, dict(src_row_stride=120), B.FCP_ERR_INVALID_ARG), ({}, dict(dst_row_stride=0), B.FCP_ERR_INVALID_ARG),
    ({}, dict(src_row_stride=132), B.FCP_ERR_UNSUPPORTED), ({}, dict(dst_row_stride=129, dst_f32=1), B.FCP_ERR_UNSUPPORTED),
    ({}, dict(src=4104), B.FCP_ERR_UNSUPPORTED), ({}, dict(dst=8194), B.FCP_ERR_UNSUPPORTED),
    ({}, dict(dst=4096, dst_row_stride=256), B.FCP_ERR_INVALID_ARG), ({}, dict(dst=4096, dst_f32=1), B.FCP_ERR_INVALID_ARG),
    ({}, dict(n_heads=2 ** 26, src_row_stride=2 ** 32, dst_row_stride=2 ** 32), B.FCP_ERR_UNSUPPORTED),
])
def test_rotary_refusals(spec, part, code):
    assert _call(spec, part) == code and B.fcp_last_error().startswith("fcp_rotary_apply")


def test_rotary_turns():
    freq = [0.0, 1.0, -1.0, 2 * np.pi, 0.25, 1e6, 1e-9]
    turn = fcp.fcp_rotary_turns(freq)
    two_pi = 2 * np.arctan(np.longdouble(1)) * 4
    for f, t in zip(freq, turn):
        want = float(np.longdouble(f) / two_pi % 1)
        assert abs((int(t) / 2.0 ** 64 - want + 0.5) % 1 - 0.5) < 1e-12 and 0 <= int(t) < 2 ** 64
    assert len(fcp.fcp_rotary_turns([])) == 0
    for bad in (float("nan"), float("inf"), -1.1e6):
        with pytest.raises(B.FcpError) as e:
            fcp.fcp_rotary_turns([0.5, bad])
        assert e.value.code == B.FCP_ERR_INVALID_ARG
    with pytest.raises(B.FcpError):
        fcp.Rotary(64, [0], [2e6])


def test_rotary_null_arguments_and_nothing_to_do():
    for null in ("r", "parts", "axis", "turn"):
        assert _call({}, {}, **{null: True}) == B.FCP_ERR_INVALID_ARG
    for n in (0, -1, 5):
        assert _call({}, {}, n) == B.FCP_ERR_INVALID_ARG
    assert _call({}, dict(n_rows=0, src=None, dst=None, pos=None), 4) == B.FCP_OK
    assert _call({}, dict(n_rows=2 ** 31 - 1, src_row_stride=120), 1) == B.FCP_ERR_INVALID_ARG


def test_rotary_binding_refuses_other_tensors():
    rot = fcp.Rotary(64, [0, 1] * 8, [0.5] * 16)
    assert rot.n_axes == 2
    x, pos = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, dtype=torch.int32)
    bad = [(x[..., :32], x, pos), (x.half(), x, pos), (x, x.double(), pos), (x[:2], x, pos), (x[:, :1], x, pos), (x, x, pos.long()), (x, x, pos[:, :1]),
           (x, x, pos.t()), (x.transpose(0, 1), x.transpose(0, 1), pos), (x[0], x[0], pos), (x, x, pos)]       # the last: not on a GPU
    for part in bad:
        with pytest.raises(ValueError):
            fcp.fcp_rotary_apply(rot, [part])
    with pytest.raises(ValueError):
        fcp.Rotary(64, [0, 1], [0.5])


def test_row_positions():
    lens, bs = [300, 40, 0, 129], 128
    plan = fcp.fcp_plan_blocks(lens, bs, 1, 0, [(0, 1), (0, 2), (3, 1)])
    q, kv = fcp.fcp_row_positions(B.Problem(plan, 2, 1, 64, bs))
    assert np.array_equal(kv, np.concatenate([np.arange(n) for n in lens]))
    assert np.array_equal(q, np.concatenate([np.arange(128, 300), [128]]))
    plan = fcp.fcp_plan_blocks_cut([10, 7], [7, 3], 4, 1, 0, [(0, 2), (1, 0), (1, 1)])
    q, kv = fcp.fcp_row_positions(B.Problem(plan, 2, 1, 64, 4))
    assert np.array_equal(kv, list(range(10)) + list(range(7))) and np.array_equal(q, [7, 8, 9] + list(range(7)))
    packed = fcp.fcp_plan_blocks_packed([5, 300, 7, 9], 128, 1, 0, None, [0, 1, 2, 3, 0, 0])
    q, kv = fcp.fcp_row_positions(B.Problem(packed, 2, 1, 64, 128))
    want = list(range(5)) + list(range(7)) + list(range(9)) + list(range(300))
    assert np.array_equal(kv, want) and np.array_equal(q, want)
    given = B.Problem(fcp.fcp_plan_blocks([200], 128, 0, 0), 2, 1, 64, 128, slopes=[1, 1], q_pos=[1000, 7], kv_pos=[50, 2000])
    q, kv = fcp.fcp_row_positions(given)
    assert np.array_equal(q, list(range(1000, 1128)) + list(range(7, 79))) and np.array_equal(kv, list(range(50, 178)) + list(range(2000, 2072)))
    assert [len(x) for x in fcp.fcp_row_positions(B.Problem(fcp.fcp_plan_blocks([], 4), 2, 1, 64, 4))] == [0, 0]


def test_row_positions_refusals():
    p = B.Problem(fcp.fcp_plan_blocks([200], 128, 1, 0), 2, 1, 64, 128)
    x = np.zeros(200, dtype=np.int32).ctypes.data
    for q, kv in ((None, x), (x, None)):
        assert B._lib.fcp_row_positions(p.ref, q, kv) == B.FCP_ERR_INVALID_ARG
    assert B._lib.fcp_row_positions(None, x, x) == B.FCP_ERR_INVALID_ARG
    plan = dict(fcp.fcp_plan_blocks([200], 128, 0, 0), q_blocks=np.array([[0, 5, 0, 128], [0, 1, 128, 72]]))
    with pytest.raises(B.FcpError):
        fcp.fcp_row_positions(B.Problem(plan, 2, 1, 64, 128))


def test_row_positions_of_plain_scores_at_given_positions():
    """Positions alone, without a softcap or slopes: a cache with gaps for rotary positions."""
    plan = fcp.fcp_plan_blocks([200], 128, 0, 0)
    p = B.Problem(plan, 2, 1, 64, 128, q_pos=[1000, 7], kv_pos=[50, 2000])
    q, kv = fcp.fcp_row_positions(p)
    assert np.array_equal(q, list(range(1000, 1128)) + list(range(7, 79))) and np.array_equal(kv, list(range(50, 178)) + list(range(2000, 2072)))
    assert B.fcp_workspace_bytes(p) == B.fcp_workspace_bytes(B.Problem(plan, 2, 1, 64, 128))       # scores stay plain
    for kw in (dict(q_pos=[0, 128]), dict(kv_pos=[0, 128]), dict(q_pos=[0, -1], kv_pos=[0, 128])):
        with pytest.raises(B.FcpError) as e:
            fcp.fcp_row_positions(B.Problem(plan, 2, 1, 64, 128, **kw))
        assert e.value.code == B.FCP_ERR_INVALID_ARG


@pytest.mark.parametrize("rows,parts", [(2 ** 26 - 3, 1), (2 ** 31 - 1, 1), (2 ** 24 - 3, 4)])
def test_rotary_refuses_more_rows_than_a_launch_holds(rows, parts):
    """2^24 workgroups of 256 threads are one more than HIP takes.  Refused in front of the launch: the pointers are never read."""
    assert _call({}, dict(n_rows=rows), parts) == B.FCP_ERR_UNSUPPORTED and "too many rows" in B.fcp_last_error()


def test_rotary_turns_are_as_good_as_stated():
    """Off by at most 1 + |freq| / 4 units of 2^-64 turns, against 2 pi in integers (Machin's formula, 2^-300)."""
    one = 1 << 300

    def arctan_inverse(n):
        total, term, k, sign = 0, one // n, 1, 1
        while term:
            total, term, k, sign = total + sign * (term // k), term // (n * n), k + 2, -sign
        return total
    two_pi = 8 * (4 * arctan_inverse(5) - arctan_inverse(239))
    rng = np.random.default_rng(0)
    freq = np.concatenate([10000.0 ** (-np.arange(64) / 64), 10.0 ** rng.uniform(-12, 6, 400) * rng.choice([-1, 1], 400), [1e6, -1e6, 2 * np.pi, np.pi]])
    for f, t in zip(freq, fcp.fcp_rotary_turns(freq)):
        num, den = float(f).as_integer_ratio()
        want = (num * one << 128) // (den * two_pi)                     # units of 2^-128 turns
        off = (((int(t) << 64) - want + (1 << 127)) % (1 << 128)) - (1 << 127)
        assert abs(off) / 2.0 ** 64 <= 1 + abs(f) / 4, f
