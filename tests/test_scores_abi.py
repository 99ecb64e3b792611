"""CPU-side checks of modified scores: the planner that cuts blocks at one more token, and every refusal."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest

import paper_2605_08524_amd as fcp
from oracle import fcp_scores_oracle as sorc
from paper_2605_08524_amd import binding as B


def _covered(plan, lens):
    """bool [T_q, T_kv] of what the pairs of a plan cover, each at most once."""
    t_q, t_kv = int(plan["q_blocks"][:, 3].sum()), int(np.sum(lens))
    n = np.zeros((t_q, t_kv), dtype=np.int32)
    for q, kv, kind, slot in plan["pairs"]:
        _, _, qs, ql = plan["q_blocks"][q]
        _, _, ks, kl = plan["kv_blocks"][kv]
        assert kind in (0, 1)
        n[qs:qs + ql, ks:ks + kl] += np.tril(np.ones((ql, kl), dtype=np.int32)) if kind else 1
        assert plan["slots"][slot][0] == q
    assert n.max(initial=0) <= 1
    return n.astype(bool)


@pytest.mark.parametrize("seed", range(40))
def test_cut_plans_cover_the_mask(seed):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 30, size=rng.integers(1, 6))
    bs = int(rng.integers(1, 9))
    cut = [int(rng.integers(0, n + 1)) for n in lens]
    prefix, c = int(rng.integers(0, 2)), int(rng.choice([0, 1, 3]))
    blocks = [(s, i) for s, n in enumerate(lens) for i in range(-(-cut[s] // bs) + -(-(int(n) - cut[s]) // bs))]
    owned = None if rng.random() < 0.4 else [b for b in blocks if rng.random() < 0.6]
    plan = fcp.fcp_plan_blocks_cut(lens, cut, bs, prefix, c, owned)
    assert [tuple(b[:2]) for b in plan["kv_blocks"]] == blocks and (plan["kv_blocks"][:, 3] <= bs).all()
    lay = sorc.layout(lens, bs, cut=cut, owned=owned)
    assert len(lay[0]) == plan["q_blocks"][:, 3].sum()
    assert np.array_equal(_covered(plan, lens), sorc.visible(*lay, mask="prefix" if prefix else "causal", cut=cut))
    rows = 0
    for s, (q, begin, n, row) in enumerate(plan["slots"]):
        assert row == rows and n == (plan["pairs"][:, 3] == s).sum() and (c == 0 or n <= c)
        rows += plan["q_blocks"][q][3]
    assert rows == plan["n_slot_rows"]
    if len(plan["pairs"]):
        B.fcp_workspace_bytes(B.Problem(plan, 2, 1, 64, bs, softcap=1.0, slopes=[1, 2]))


@pytest.mark.parametrize("prefix", [0, 1])
def test_a_cut_at_nothing_is_the_plain_causal_plan(prefix):
    lens = [300, 0, 77, 512]
    a, b = fcp.fcp_plan_blocks(lens, 128, 1, 2), fcp.fcp_plan_blocks_cut(lens, [0] * 4, 128, prefix, 2)
    for key in ("kv_blocks", "q_blocks", "pairs", "slots", "n_slot_rows"):
        assert np.array_equal(a[key], b[key])
    b = fcp.fcp_plan_blocks_cut(lens, [256, 0, 0, 128], 128, 0, 2)
    assert np.array_equal(a["pairs"], b["pairs"])
    whole = fcp.fcp_plan_blocks_cut(lens, lens, 128, 1, 2)                  # all of it a prefix: a full mask
    full = fcp.fcp_plan_blocks(lens, 128, 0, 2)
    for key in ("kv_blocks", "q_blocks", "pairs", "slots"):
        assert np.array_equal(whole[key], full[key])


@pytest.mark.parametrize("args,code", [
    (([5], [6], 4), B.FCP_ERR_INVALID_ARG), (([5], [-1], 4), B.FCP_ERR_INVALID_ARG), (([-5], [0], 4), B.FCP_ERR_INVALID_ARG),
    (([5], [1], 0), B.FCP_ERR_INVALID_ARG), (([5], [1], 4, 0, -1), B.FCP_ERR_INVALID_ARG),
    (([5], [1], 4, 0, 0, [(0, 2)]), B.FCP_ERR_INVALID_ARG), (([5], [1], 4, 0, 0, [(0, 1), (0, 0)]), B.FCP_ERR_INVALID_ARG),
    (([2 ** 30, 2 ** 30], [1, 1], 2 ** 30), B.FCP_ERR_UNSUPPORTED),
])
def test_cut_planner_refusals(args, code):
    with pytest.raises(B.FcpError) as e:
        fcp.fcp_plan_blocks_cut(*args)
    assert e.value.code == code


def test_cut_planner_capacities_and_null():
    lib, n = B._lib, [C.c_int32(0) for _ in range(5)]
    i32p = C.POINTER(C.c_int32)
    lens, cut = (np.asarray(x, dtype=np.int32).ctypes.data_as(i32p) for x in ([9], [3]))
    none = [None, C.byref(n[0]), None, C.byref(n[1]), None, C.byref(n[2]), None, C.byref(n[3]), C.byref(n[4])]
    assert lib.fcp_plan_blocks_cut(lens, None, 1, 4, 0, 0, None, 0, *none) == B.FCP_ERR_INVALID_ARG
    assert lib.fcp_plan_blocks_cut(lens, cut, 1, 4, 0, 0, None, 0, *none) == B.FCP_OK
    want = [x.value for x in n]
    assert want[:4] == [3, 3, 6, 3]
    tabs = [np.zeros((x, 4), dtype=np.int32) for x in want[:4]]
    n[2].value -= 1
    call = [a for t, x in zip(tabs, n) for a in (t.ctypes.data, C.byref(x))] + [C.byref(n[4])]
    assert lib.fcp_plan_blocks_cut(lens, cut, 1, 4, 0, 0, None, 0, *call) == B.FCP_ERR_BUFFER_TOO_SMALL and n[2].value == want[2]
    with pytest.raises(ValueError):
        fcp.fcp_plan_blocks_cut([3, 4], [1], 4)


def _problem(plan=None, hq=2, **kw):
    return B.Problem(plan or fcp.fcp_plan_blocks([300, 40], 128, 1, 2), hq, 1, 64, 128, **kw)


def test_scores_accepted():
    plain = B.fcp_workspace_bytes(_problem())
    assert B.fcp_workspace_bytes(_problem(softcap=30.0)) == plain                 # a cap needs no table
    assert B.fcp_workspace_bytes(_problem(slopes=[0.5, 0.0])) > plain
    assert _problem().flags & B.FCP_FLAG_SCORES == 0 and _problem(softcap=1.0).flags & B.FCP_FLAG_SCORES
    for cap in (2.0 ** -10, 1024.0):
        B.fcp_workspace_bytes(_problem(softcap=cap))
    p = _problem(flags=B.FCP_FLAG_SCORES)                                         # neither: plain scores
    assert B.fcp_workspace_bytes(p) == plain


@pytest.mark.parametrize("kw", [
    dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=float("inf")), dict(softcap=1025.0), dict(softcap=2.0 ** -11),
    dict(slopes=[0.5, -0.5]), dict(slopes=[0.5, float("nan")]), dict(slopes=[float("inf"), 0]), dict(slopes=[1e30, 0]),
    dict(slopes=[1, 1], q_pos=[0, 128, 256, 0]), dict(slopes=[1, 1], kv_pos=[0, 128, 256, 0]),
    dict(slopes=[1, 1], q_pos=[0, 128, -1, 0], kv_pos=[0, 128, 256, 0]), dict(slopes=[1, 1], q_pos=[0, 128, 256, 0], kv_pos=[0, 128, 2 ** 31 - 10, 0]),
])
def test_scores_refused_by_every_call(kw):
    p = _problem(**kw)
    x = 4096        # never read: the call ends before
    calls = [lambda: B.fcp_workspace_bytes(p), lambda: B.fcp_queue_build(p, x, 1 << 30), lambda: B.fcp_block_attn_fwd(p, x, x, x, x, x, x),
             lambda: B.fcp_block_attn_fwd_out(p, x, x, x, x, x, x, x, x), lambda: B.fcp_block_attn_fwd_static(p, x, x, x, x, x),
             lambda: B.fcp_merge_partials(p, x, x, x, x, x), lambda: B.fcp_block_attn_bwd(p, x, x, x, x, x, x, x, x, x, x),
             lambda: B.fcp_block_attn_bwd_dkdv(p, x, x, x, x, x, x, x), lambda: B.fcp_block_attn_bwd_dq(p, x, x, x, x, x, x), lambda: B.fcp_launch_probe(p)]
    for call in calls:
        with pytest.raises(B.FcpError) as e:
            call()
        assert e.value.code == B.FCP_ERR_INVALID_ARG and "scores" in str(e.value)


def test_small_prefix_launches_are_split_like_causal_ones():
    lens, cut = [4000], [2000]
    for kw in ({}, dict(softcap=20.0, slopes=[0.1] * 4)):
        probes = [fcp.fcp_launch_probe(B.Problem(p, 4, 4, 64, 512, **kw)) for p in (fcp.fcp_plan_blocks_cut(lens, cut, 512, 1, 0), fcp.fcp_plan_blocks(lens, 512, 1, 0))]
        assert probes[0]["split"] == probes[1]["split"] == (True, True, True)
    # a stage of such a plan is not known to be all that its rows see
    stage, _ = fcp.fcp_stage_tables(fcp.fcp_plan_blocks_cut([4000], [4000], 512, 1, 8), 0)
    assert not fcp.fcp_launch_probe(B.Problem(stage, 16, 16, 64, 512, flags=B.FCP_FLAG_RUNNING_MERGE | B.FCP_FLAG_O_F32))["split"][0]


def test_scores_null_and_argument_lengths():
    p = _problem(softcap=1.0)
    p.c.scores = None
    with pytest.raises(B.FcpError) as e:
        B.fcp_workspace_bytes(p)
    assert e.value.code == B.FCP_ERR_INVALID_ARG
    for kw in (dict(slopes=[1.0]), dict(slopes=[1, 1], q_pos=[0], kv_pos=[0, 128, 256, 0]), dict(slopes=[1, 1], q_pos=[0, 128, 256, 0], kv_pos=[0])):
        with pytest.raises(ValueError):
            _problem(**kw)


def test_positions_that_the_tables_do_not_give():
    plan = fcp.fcp_plan_blocks([300], 128, 1, 0, [(0, 2)])
    far = dict(plan, q_blocks=np.array([[0, 7, 0, 44]], dtype=np.int32), pairs=np.array([[0, 0, 0, 0], [0, 1, 0, 0]], dtype=np.int32),
               slots=np.array([[0, 0, 2, 0]], dtype=np.int32))
    B.fcp_workspace_bytes(_problem(far, softcap=3.0))                             # no positions needed
    with pytest.raises(B.FcpError):
        B.fcp_workspace_bytes(_problem(far, slopes=[1, 1]))
    B.fcp_workspace_bytes(_problem(far, slopes=[1, 1], q_pos=[900], kv_pos=[0, 128, 256]))
    other = fcp.fcp_plan_blocks([128, 128], 128, 0, 0)
    other["pairs"][1][1] = 0                                                      # a row block of one sequence on keys of another
    with pytest.raises(B.FcpError):
        B.fcp_workspace_bytes(_problem(other, slopes=[1, 1]))
    B.fcp_workspace_bytes(_problem(other, slopes=[1, 1], q_pos=[0, 128], kv_pos=[0, 128]))


def test_a_diagonal_pair_is_at_one_position():
    plan = fcp.fcp_plan_blocks([200], 128, 1, 0)
    B.fcp_workspace_bytes(_problem(plan, slopes=[1, 1], q_pos=[50, 178], kv_pos=[50, 178]))
    for q_pos in ([51, 178], [50, 100]):
        with pytest.raises(B.FcpError) as e:
            B.fcp_workspace_bytes(_problem(plan, slopes=[1, 1], q_pos=q_pos, kv_pos=[50, 178]))
        assert e.value.code == B.FCP_ERR_INVALID_ARG and "scores" in str(e.value)
    # a KV block that is there twice: the second is behind the first, its query block at the first
    twice = dict(fcp.fcp_plan_blocks([100], 128, 1, 0), kv_blocks=np.array([[0, 0, 0, 100], [0, 0, 100, 100]], dtype=np.int32))
    B.fcp_workspace_bytes(_problem(twice, slopes=[1, 1]))
    twice["pairs"] = np.array([[0, 1, 1, 0]], dtype=np.int32)
    with pytest.raises(B.FcpError):
        B.fcp_workspace_bytes(_problem(twice, slopes=[1, 1]))
    # all keys of a full pair are seen, wherever they are
    B.fcp_workspace_bytes(_problem(fcp.fcp_plan_blocks([200], 128, 0, 0), slopes=[1, 1], q_pos=[7, 3], kv_pos=[50, 178]))


def test_the_largest_slopes():
    B.fcp_workspace_bytes(_problem(slopes=[64.0, 0.0], softmax_scale=1e-20))
    for kw in (dict(slopes=[0.0, np.nextafter(np.float32(64), np.float32(65))]), dict(slopes=[64.0, 0.0], softmax_scale=1e-21)):
        with pytest.raises(B.FcpError) as e:
            B.fcp_workspace_bytes(_problem(**kw))
        assert e.value.code == B.FCP_ERR_INVALID_ARG and "scores" in str(e.value)


def test_a_host_without_memory_is_an_error_not_an_abort():
    """In a child whose address space is as large as it is: tables of 4 million blocks need more."""
    code = """
import resource, sys
import numpy as np
sys.path.insert(0, %r)
import paper_2605_08524_amd as fcp
from paper_2605_08524_amd import binding as B
n = 4000000
lens = np.ones(n, dtype=np.int32)
plan = fcp.fcp_plan_blocks(lens, 1, 1, 0)
p = B.Problem(plan, 2, 1, 64, 1, slopes=[1, 1])
x = np.zeros(n, dtype=np.int32)
size = int(open('/proc/self/statm').read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (size + (8 << 20),) * 2)
for call in (lambda: B.fcp_workspace_bytes(p), lambda: fcp.fcp_row_positions(p), lambda: B.fcp_block_attn_fwd(p, 1, 1, 1, 1, 1, 256)):
    try:
        call()
    except B.FcpError as e:
        assert e.code == B.FCP_ERR_UNSUPPORTED and 'memory' in str(e), e
    except MemoryError:
        pass
    else:
        raise SystemExit('no error')
print('fine')
""" % os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "fine" in r.stdout, (r.returncode, r.stderr[-500:])


def test_slopes_need_a_workspace_that_was_built_with_them():
    """A workspace that nothing was built into may have been built without slopes: too small for a layout that has them."""
    p = _problem(slopes=[0.5, 0.25])
    x = 4096        # never read: the call ends before
    for call in (lambda: B.fcp_block_attn_fwd(p, x, x, x, x, x, x), lambda: B.fcp_block_attn_fwd_out(p, x, x, x, x, x, x, x, x),
                 lambda: B.fcp_merge_partials(p, x, x, x, x, x), lambda: B.fcp_bwd_preprocess(p, x, x, x, x), lambda: B.fcp_block_attn_bwd(p, x, x, x, x, x, x, x, x, x, x),
                 lambda: B.fcp_block_attn_bwd_dkdv(p, x, x, x, x, x, x, x), lambda: B.fcp_block_attn_bwd_dq(p, x, x, x, x, x, x),
                 lambda: B.fcp_block_attn_bwd_dq_d(p, x, x, x, x, x, x, x, x)):
        with pytest.raises(B.FcpError) as e:
            call()
        assert e.value.code == B.FCP_ERR_INVALID_ARG and "slopes" in str(e.value)
