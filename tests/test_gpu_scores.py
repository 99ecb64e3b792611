"""GPU parity of modified scores (softcap, distance bias, prefix masks, with packed documents, stages, shares and single tokens)
against the fp64 oracle.  Every element of every output is held to a bound that the oracle derives for it: bf16 roundings of P, dS, O and
gradients at half a step each, fp32 for the rest.  Both families of kernels run: the split ones that small launches choose, and
(FCP_FLAG_WHOLE_ITEMS) those of large launches."""
import numpy as np
import pytest
import torch

import paper_2605_08524_amd as fcp
from oracle import fcp_oracle as orc
from oracle import fcp_scores_oracle as sorc
from paper_2605_08524_amd import workloads

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BASE = fcp.FCP_FLAG_DIRECT_SINGLE | fcp.FCP_FLAG_O_F32


def alibi(hq):
    return [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]


def bits_to_dev(bits):
    return torch.from_numpy(bits.view(np.int16)).to(DEV).view(torch.bfloat16)


class Run:
    """A problem with its device buffers; outputs start as NaN."""

    def __init__(self, plan, hq, hkv, d, bs, flags=BASE, backward=True, seed=0, q_scale=1.0, **kw):
        self.p = p = fcp.Problem(plan, hq, hkv, d, bs, 0.0, flags, **kw)
        self.bits = [workloads.draw_tensor(seed, i + 1, (n, h, d)) for i, (n, h) in enumerate(((p.t_q, hq), (p.t_kv, hkv), (p.t_kv, hkv), (p.t_q, hq)))]
        if q_scale != 1.0:
            self.bits[0] = workloads.bf16_bits(workloads.bf16_to_f32(self.bits[0]) * np.float32(q_scale))
        self.q, self.k, self.v, self.d_o = (bits_to_dev(b) for b in self.bits)
        nan = float("nan")
        full = lambda shape, dt=torch.float32: torch.full(shape, nan, dtype=dt, device=DEV)
        g = torch.bfloat16 if flags & fcp.FCP_FLAG_GRAD_BF16 else torch.float32
        self.o = full((p.t_q, hq, d), torch.float32 if flags & fcp.FCP_FLAG_O_F32 else torch.bfloat16)
        self.lse = full((p.t_q, hq))
        self.o_part, self.lse_part = full((max(1, p.n_slot_rows), hq, d)), full((max(1, p.n_slot_rows), hq))
        self.dq, self.dk, self.dv = full((p.t_q, hq, d), g), full((p.t_kv, hkv, d), g), full((p.t_kv, hkv, d), g)
        n = fcp.fcp_workspace_bytes(p)
        self.ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device=DEV)
        self.ws_ptr = self.ws.data_ptr() + (-self.ws.data_ptr()) % 256
        fcp.fcp_queue_build(p, self.ws_ptr, n)
        self.backward = backward

    def step(self, stream=None):
        fcp.fcp_block_attn_fwd_out(self.p, self.q, self.k, self.v, self.o_part, self.lse_part, self.o, self.lse, self.ws_ptr, stream)
        fcp.fcp_merge_partials(self.p, self.o_part, self.lse_part, self.o, self.lse, self.ws_ptr, stream)
        if self.backward:
            fcp.fcp_block_attn_bwd(self.p, self.q, self.k, self.v, self.o, self.lse, self.d_o, self.dq, self.dk, self.dv, self.ws_ptr, stream)

    def outputs(self):
        names = ("o", "lse", "dq", "dk", "dv") if self.backward else ("o", "lse")
        torch.cuda.synchronize()
        return {n: getattr(self, n).double().cpu().numpy() for n in names}

    def check(self, see, dist, got=None):
        got = got or self.outputs()
        p = self.p
        q, k, v, do = (orc.bf16_to_f64(b) for b in self.bits)
        want = sorc.attention(q, k, v, see, dist, p.softcap, p.slopes, None, do if self.backward else None,
                              o_bf16=not p.flags & fcp.FCP_FLAG_O_F32, grad_bf16=bool(p.flags & fcp.FCP_FLAG_GRAD_BF16))
        for name, x in got.items():
            ref, bound = want[name]
            if name == "lse":
                assert np.array_equal(np.isneginf(x), np.isneginf(ref))
                x, ref, bound = (y[np.isfinite(ref)] for y in (x, ref, bound))
            assert np.isfinite(x).all(), name
            err = np.abs(x - ref)
            worst = float((err / bound).max(initial=0))
            print(f"  {name}: worst {worst:.2f} of its bound, max-abs {err.max(initial=0):.2e}", flush=True)
            assert worst <= 1.0, (name, worst)


def geometry(lay, mask="causal", cut=None):
    return sorc.visible(*lay, mask=mask, cut=cut), np.abs(lay[1][:, None] - lay[3][None])


GEOMETRY = {
    # lens, block, mask, cut, coalesce, Hq, Hkv, d, owned
    "one_token": ([1], 64, "causal", None, 0, 4, 2, 64, None),
    "ragged": ([300, 77, 129, 1], 128, "causal", None, 2, 4, 2, 64, None),
    "ragged_d128": ([290, 65, 64, 2], 128, "causal", None, 1, 2, 1, 128, None),
    "odd_group": ([333, 31], 100, "causal", None, 3, 6, 2, 64, None),
    "odd_group_d128": ([400], 256, "causal", None, 0, 3, 1, 128, None),
    "full": ([260, 90], 128, "full", None, 2, 4, 4, 64, None),
    "full_d128": ([260, 90], 64, "full", None, 16, 8, 2, 128, None),
    "prefix": ([300, 200, 90, 64], 128, "prefix", [130, 0, 90, 63], 2, 4, 2, 64, None),
    "prefix_d128": ([270, 140], 128, "prefix", [1, 128], 0, 4, 1, 128, None),
    "decode": ([700, 1, 257, 128], 128, "causal", [699, 0, 256, 127], 2, 8, 2, 64, [(0, 6), (1, 0), (2, 2), (3, 1)]),
    "decode_d128": ([900, 300], 256, "causal", [899, 299], 1, 4, 4, 128, [(0, 4), (1, 2)]),
    "chunk": ([500, 80], 128, "causal", [430, 10], 2, 4, 2, 64, [(0, 4), (1, 1)]),
    "share": ([700], 128, "causal", None, 2, 4, 1, 64, [(0, 0), (0, 2), (0, 5)]),
    "share_d128": ([600, 50], 128, "causal", None, 4, 2, 2, 128, [(0, 1), (0, 4), (1, 0)]),
    # more than eight KV tiles an item
    "long": ([1500, 700], 512, "causal", None, 0, 4, 2, 64, None),
    "long_d128": ([1100], 256, "causal", None, 3, 2, 1, 128, None),
    "long_odd_group": ([1300, 577], 384, "causal", None, 0, 3, 1, 64, None),
    "long_full": ([900, 650], 512, "full", None, 0, 2, 1, 64, None),
    "long_prefix": ([1400, 800], 512, "prefix", [900, 333], 0, 4, 4, 64, None),
    "long_prefix_d128": ([1200], 300, "prefix", [700], 4, 2, 1, 128, None),
    "short_rows": ([40, 64, 9, 33, 60], 64, "causal", None, 0, 8, 2, 128, None),
}
SCORES = {"bias": (0.0, True), "cap": (20.0, False), "both": (5.0, True), "wide": (400.0, True), "wide_cap": (90.0, False)}


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", SCORES)
@pytest.mark.parametrize("geo", GEOMETRY)
def test_forward_and_backward(geo, scores, whole):
    lens, bs, mask, cut, c, hq, hkv, d, owned = GEOMETRY[geo]
    cap, bias = SCORES[scores]
    if cut is None:
        plan = fcp.fcp_plan_blocks(lens, bs, int(mask == "causal"), c, owned)
    else:
        plan = fcp.fcp_plan_blocks_cut(lens, cut, bs, int(mask == "prefix"), c, owned)
    # alternate what the backward does and how it writes
    n = list(GEOMETRY).index(geo) + list(SCORES).index(scores)
    flags = BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0) | (fcp.FCP_FLAG_BWD_SPILL_DS if n % 2 else 0) | (fcp.FCP_FLAG_GRAD_BF16 if n % 3 == 0 else 0)
    run = Run(plan, hq, hkv, d, bs, flags, seed=n, q_scale=4.0, softcap=cap, slopes=alibi(hq) if bias else None)
    run.step()
    run.check(*geometry(sorc.layout(lens, bs, cut=cut, owned=owned), mask, cut))


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", ["bias", "cap", "both"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (3, 3, 128)])
def test_documents_that_share_blocks(hq, hkv, d, causal, scores, whole):
    lens = [5, 60, 1, 130, 17, 33, 100, 2, 40, 128, 70]
    units, room, bs = [], 0, 256
    for n in lens:
        if n > room:
            units.append((units[-1] + 1) if units else 0)
            room = bs
        else:
            units.append(units[-1])
        room -= n
    plan = fcp.fcp_plan_blocks_packed(lens, bs, causal, 0, None, units)
    assert len(plan["segments"])
    cap, bias = SCORES[scores]
    for spill in (0, fcp.FCP_FLAG_BWD_SPILL_DS):
        run = Run(plan, hq, hkv, d, bs, BASE | spill | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=7, q_scale=3.0, softcap=cap, slopes=alibi(hq) if bias else None)
        run.step()
        run.check(*geometry(sorc.layout(lens, bs), "causal" if causal else "full"))


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", ["bias", "both"])
def test_steep_slopes_and_far_partials(scores, whole):
    """Slopes that leave next to nothing but the own token; partial slots far away have an LSE of -1000s and still their own maximum."""
    lens, bs, hq = [1000], 64, 4
    slopes = [40.0, 3.0, 0.7, 0.0]
    plan = fcp.fcp_plan_blocks(lens, bs, 1, 2)
    run = Run(plan, hq, 2, 64, bs, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=3, softcap=SCORES[scores][0], slopes=slopes)
    run.step()
    lay = sorc.layout(lens, bs)
    see, dist = geometry(lay)
    run.check(see, dist)
    # every partial against the oracle over its own columns
    torch.cuda.synchronize()
    q, k, v, _ = (orc.bf16_to_f64(b) for b in run.bits)
    qb, kb = plan["q_blocks"], plan["kv_blocks"]
    n_slots = {b: (plan["slots"][:, 0] == b).sum() for b in range(len(qb))}
    for s, (b, begin, n, row) in enumerate(plan["slots"]):
        if n_slots[b] == 1:
            continue                     # written to the final output
        kvs = plan["pairs"][begin:begin + n, 1]
        rows, cols = slice(qb[b][2], qb[b][2] + qb[b][3]), slice(kb[kvs[0]][2], kb[kvs[-1]][2] + kb[kvs[-1]][3])
        want = sorc.attention(q[rows], k[cols], v[cols], see[rows, cols], dist[rows, cols], run.p.softcap, run.p.slopes)
        for name, x in (("o", run.o_part), ("lse", run.lse_part)):
            got = x[row:row + qb[b][3]].double().cpu().numpy()
            ref, bound = want[name]
            assert np.array_equal(np.isneginf(got), np.isneginf(ref))
            assert (np.abs(got - ref)[np.isfinite(ref)] <= bound[np.isfinite(ref)]).all(), (s, name)


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("cap", [0.0625, 4.0, 50.0, 60.0, 1024.0])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_far_beyond_the_cap(cap, d, whole):
    """Logits of hundreds: tanh saturates both ways, in rows whose scores are all low and rows whose scores are all high."""
    lens, bs = [200, 70], 128
    plan = fcp.fcp_plan_blocks(lens, bs, 1, 1)
    run = Run(plan, 2, 1, d, bs, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=11, q_scale=1.0, softcap=cap)
    k0 = workloads.bf16_to_f32(run.bits[1])
    k0[:, 0, :8] = 6.0                                    # a direction that all keys share
    q0 = workloads.bf16_to_f32(run.bits[0])
    q0[0::3, :, :8], q0[1::3, :, :8] = 40.0, -40.0
    run.bits[0], run.bits[1] = workloads.bf16_bits(q0), workloads.bf16_bits(k0)
    run.q, run.k = bits_to_dev(run.bits[0]), bits_to_dev(run.bits[1])
    run.step()
    run.check(*geometry(sorc.layout(lens, bs)))


@pytest.mark.parametrize("scores", ["bias", "both"])
@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
def test_positions_given_by_the_caller(scores, whole):
    """Tables with gaps: KV blocks of a sequence that are not all there, in another order than the pairs', and a query token whose block
    is none of them (FULL pairs only, as a token behind a cache has)."""
    kv = [(0, 0, 100), (0, 2, 64), (0, 3, 128), (0, 9, 30)]          # seq, idx, tokens
    kv_pos, q_pos, q_len = [0, 200, 264, 5000], [5030, 264], [1, 128]
    start = np.concatenate([[0], np.cumsum([n for _, _, n in kv])])
    plan = dict(kv_blocks=[(s, i, start[n], ln) for n, (s, i, ln) in enumerate(kv)], q_blocks=[(0, 10, 0, 1), (0, 3, 1, 128)],
                pairs=[(0, 0, 0, 0), (0, 2, 0, 0), (0, 1, 0, 0), (0, 3, 0, 1), (1, 1, 0, 2), (1, 0, 0, 2), (1, 2, 1, 2)],
                slots=[(0, 0, 3, 0), (0, 3, 1, 1), (1, 4, 3, 2)], n_slot_rows=130)
    cap, _ = SCORES[scores]
    run = Run(plan, 4, 2, 64, 128, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=5, softcap=cap, slopes=[0.25, 0.01, 0.001, 0.0], q_pos=q_pos, kv_pos=kv_pos)
    run.step()
    kp = np.concatenate([p + np.arange(n) for p, (_, _, n) in zip(kv_pos, kv)])
    qp = np.concatenate([p + np.arange(n) for p, n in zip(q_pos, q_len)])
    see = np.ones((129, len(kp)), dtype=bool)
    see[1:, start[3]:] = False
    see[1:, start[2]:start[3]] = np.tril(np.ones((128, 128), dtype=bool))
    run.check(see, np.abs(qp[:, None] - kp[None]))


@pytest.mark.parametrize("scores", ["bias", "cap", "both", "wide"])
@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
def test_slots_of_many_scattered_spans(scores, whole):
    """Slots whose KV blocks do not follow each other: every block a span of its own, ragged ends between them, more than 64 of them."""
    rng = np.random.default_rng(4)
    kv_len = [int(n) for n in rng.integers(1, 40, size=150)]
    kv_pos = [int(x) for x in rng.integers(0, 30000, size=150)]
    start = np.concatenate([[0], np.cumsum(kv_len)])
    q_len, q_pos = [40, 1, 33], [9000, 30000, 100]
    pairs, slots, row = [], [], 0
    see = np.zeros((74, start[-1]), dtype=bool)
    q0 = 0
    for b, (n, count) in enumerate(zip(q_len, (100, 140, 7))):
        slots.append((b, len(pairs), count, row))
        for j in rng.permutation(150)[:count]:
            pairs.append((b, j, 0, b))
            see[q0:q0 + n, start[j]:start[j + 1]] = True
        row, q0 = row + n, q0 + n
    plan = dict(kv_blocks=[(0, i, start[i], n) for i, n in enumerate(kv_len)], q_blocks=[(0, 200 + b, s, n) for b, (s, n) in enumerate(zip((0, 40, 41), q_len))],
                pairs=pairs, slots=slots, n_slot_rows=74)
    cap, bias = SCORES[scores]
    run = Run(plan, 4, 2, 64, 64, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=12, q_scale=2.0, softcap=cap,
              slopes=[0.25, 0.001, 0.0001, 0.0] if bias else None, q_pos=q_pos, kv_pos=kv_pos)
    run.step()
    kp = np.concatenate([p + np.arange(n) for p, n in zip(kv_pos, kv_len)])
    qp = np.concatenate([p + np.arange(n) for p, n in zip(q_pos, q_len)])
    run.check(see, np.abs(qp[:, None] - kp[None]))


def test_rows_without_keys_and_far_positions():
    """A query block without a slot, and positions close to 2^31."""
    plan = fcp.fcp_plan_blocks([256], 128, 1, 0)
    plan["pairs"], plan["slots"], plan["n_slot_rows"] = np.array([[1, 0, 0, 0], [1, 1, 1, 0]]), np.array([[1, 0, 2, 0]]), 128
    top = 2 ** 31 - 1 - 256
    run = Run(plan, 2, 2, 64, 128, BASE, seed=9, softcap=10.0, slopes=[0.5, 0.125], q_pos=[top, top + 128], kv_pos=[top, top + 128])
    run.step()
    lay = sorc.layout([256], 128)
    see, dist = geometry(lay)
    see[:128] = False
    run.check(see, dist)


@pytest.mark.parametrize("scores", SCORES)
def test_stages_with_a_running_result(scores):
    lens, bs, c = [500, 130], 64, 2
    cap, bias = SCORES[scores]
    kw = dict(softcap=cap, slopes=alibi(4) if bias else None)
    plan = fcp.fcp_plan_blocks(lens, bs, 1, c)
    ref = Run(plan, 4, 2, 64, bs, BASE, backward=False, seed=2, **kw)
    o, lse = torch.full_like(ref.o, float("nan")), torch.full_like(ref.lse, float("-inf"))
    for st in range(fcp.fcp_stage_tables(plan, 0)[1]):
        stage, _ = fcp.fcp_stage_tables(plan, st)
        p = fcp.Problem(stage, 4, 2, 64, bs, 0.0, fcp.FCP_FLAG_RUNNING_MERGE | fcp.FCP_FLAG_O_F32, **kw)
        n = fcp.fcp_workspace_bytes(p)
        ws = torch.empty(n + 256, dtype=torch.uint8, device=DEV)
        ptr = ws.data_ptr() + (-ws.data_ptr()) % 256
        fcp.fcp_queue_build(p, ptr, n)
        fcp.fcp_block_attn_fwd_out(p, ref.q, ref.k, ref.v, None, None, o, lse, ptr)
        torch.cuda.synchronize()
    ref.check(*geometry(sorc.layout(lens, bs)), got={"o": o.double().cpu().numpy(), "lse": lse.double().cpu().numpy()})


@pytest.mark.parametrize("scores", SCORES)
@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 2), (128, 3, 1)])
def test_static_forward_and_stage_calls_agree_bit_for_bit(scores, d, hq, hkv):
    cap, bias = SCORES[scores]
    kw = dict(softcap=cap, slopes=alibi(hq) if bias else None)
    plan = fcp.fcp_plan_blocks([400, 90], 128, 1, 2)
    for spill in (0, fcp.FCP_FLAG_BWD_SPILL_DS):
        run = Run(plan, hq, hkv, d, 128, fcp.FCP_FLAG_O_F32 | spill, seed=4, q_scale=3.0, **kw)
        run.step()
        first = run.outputs()
        op, lp = torch.full_like(run.o_part, float("nan")), torch.full_like(run.lse_part, float("nan"))
        fcp.fcp_block_attn_fwd_static(run.p, run.q, run.k, run.v, op, lp)
        torch.cuda.synchronize()
        assert torch.equal(op, run.o_part) and torch.equal(lp, run.lse_part)
        for x in (run.dq, run.dk, run.dv):
            x.fill_(float("nan"))
        fcp.fcp_bwd_preprocess(run.p, run.o, run.lse, run.d_o, run.ws_ptr)
        fcp.fcp_block_attn_bwd_dkdv(run.p, run.q, run.k, run.v, run.d_o, run.dk, run.dv, run.ws_ptr)
        if spill:
            fcp.fcp_block_attn_bwd_dq_ds(run.p, run.k, run.dq, run.ws_ptr)
        else:
            fcp.fcp_block_attn_bwd_dq(run.p, run.q, run.k, run.v, run.d_o, run.dq, run.ws_ptr)
        for name, x in run.outputs().items():
            assert np.allclose(x, first[name], rtol=0, atol=1e-5) if name == "dq" else np.array_equal(x, first[name]), name


@pytest.mark.parametrize("scores", ["bias", "cap", "both"])
def test_a_step_replays_from_a_graph_on_another_stream(scores):
    cap, bias = SCORES[scores]
    plan = fcp.fcp_plan_blocks([900, 300, 40], 128, 1, 2)
    run = Run(plan, 4, 2, 64, 128, BASE, seed=6, q_scale=2.0, softcap=cap, slopes=alibi(4) if bias else None)
    run.step()
    eager = run.outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run.step(side)
    for _ in range(3):
        for x in (run.o, run.lse, run.dq, run.dk, run.dv):
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        got = run.outputs()
        for name, x in got.items():
            assert np.array_equal(x, eager[name]), name
        run.step()                       # the program's own eager step in between
        for name, x in run.outputs().items():
            assert np.array_equal(x, eager[name]), name


def test_slopes_of_zero_and_a_cap_out_of_reach_change_little():
    """Zero slopes are plain scores but for what P is rounded against (half a step of bf16 each way, so twice the oracle's bound between two
    results that each keep to it); a cap of 1024 on small scores is one to 1e-4."""
    lens, bs = [500, 77], 128
    plan = fcp.fcp_plan_blocks(lens, bs, 1, 2)
    runs = [Run(plan, 4, 2, 64, bs, BASE, seed=8, **kw) for kw in ({}, dict(slopes=[0.0] * 4), dict(softcap=1024.0))]
    see, dist = geometry(sorc.layout(lens, bs))
    for r in runs:
        r.step()
        r.check(see, dist)
    plain, _, capped = (r.outputs() for r in runs)
    for name in plain:
        # tanh(x) = x - x^3 / 3: scores of up to 6 lose 6^3 / (3 1024^2) = 7e-5 of themselves, P and the outputs as much, and roundings may differ
        assert np.abs(capped[name] - plain[name]).max() <= 2.0 ** -7 * np.abs(plain[name]).max(), name


def test_a_workspace_built_without_slopes_is_refused_and_one_with_them_serves_plain_scores():
    plan = fcp.fcp_plan_blocks([300, 40], 128, 1, 2)
    plain, biased = (Run(plan, 2, 1, 64, 128, BASE, seed=1, **kw) for kw in ({}, dict(slopes=[0.5, 0.1])))
    with pytest.raises(fcp.FcpError) as e:
        fcp.fcp_block_attn_fwd_out(biased.p, plain.q, plain.k, plain.v, plain.o_part, plain.lse_part, plain.o, plain.lse, plain.ws_ptr)
    assert e.value.code == -1 and "slopes" in str(e.value)
    plain.step()
    want = plain.outputs()
    plain.ws_ptr = biased.ws_ptr
    for x in (plain.o, plain.lse, plain.dq, plain.dk, plain.dv):
        x.fill_(float("nan"))
    plain.step()
    for name, x in plain.outputs().items():
        assert np.array_equal(x, want[name]), name


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("cap", [59.0, 60.3, 60.5, 100.0])
def test_rows_whose_scores_are_all_at_one_end_of_the_cap(cap, whole):
    """Every score of a row at -cap (or +cap), values down to 2^-20: what the fixed reference leaves of the exponent range must do for them."""
    lens, bs = [300], 128
    plan = fcp.fcp_plan_blocks(lens, bs, 0, 1)
    run = Run(plan, 2, 1, 64, bs, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=13, softcap=cap)
    q, k, v = (workloads.bf16_to_f32(b) for b in run.bits[:3])
    q[:], k[:] = 0.0, 0.0
    k[..., 0] = 64.0
    q[0::2, :, 0], q[1::2, :, 0] = -64.0, 64.0                # z = +-512
    v *= np.float32(2.0) ** -np.random.default_rng(0).integers(0, 21, size=v.shape).astype(np.float32)
    for i, x in enumerate((q, k, v)):
        run.bits[i] = workloads.bf16_bits(x)
    run.q, run.k, run.v = (bits_to_dev(b) for b in run.bits[:3])
    run.step()
    got = run.outputs()
    run.check(*geometry(sorc.layout(lens, bs), "full"), got=got)
    # equal scores: the mean of V, every column to a bf16 rounding of its own size
    mean = np.abs(orc.bf16_to_f64(run.bits[2])).mean(0)
    assert (np.abs(got["o"] - orc.bf16_to_f64(run.bits[2]).mean(0)[None]) <= 2.0 ** -7 * mean[None]).all()


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", ["bias", "both", "wide"])
@pytest.mark.parametrize("d,lens", [(64, [300, 129]), (128, [1100])])
def test_the_steepest_slopes_keep_the_own_token_s_score(d, lens, scores, whole):
    """Under a slope of 64 the own token is all that a row sees, and its LSE the own score: no multiple of the slope may be left of a bias that is 0
    there.  Its line over the columns of a tile is off by half a unit of 64 slopes (2^-18 of a slope), twice: where it starts and where it is added."""
    slopes = [64.0, 63.9]
    plan = fcp.fcp_plan_blocks(lens, 256, 1, 0)
    run = Run(plan, 2, 1, d, 256, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), backward=False, seed=13, softcap=SCORES[scores][0], slopes=slopes)
    run.step()
    lay = sorc.layout(lens, 256)
    see, dist = geometry(lay)
    q, k, v, _ = (orc.bf16_to_f64(b) for b in run.bits)
    _, plain = sorc.attention(q, k, v, np.eye(len(q), dtype=bool), dist, run.p.softcap, None)["lse"]     # what fp32 does to the own score
    want, _ = sorc.attention(q, k, v, see, dist, run.p.softcap, run.p.slopes)["lse"]
    err = np.abs(run.outputs()["lse"] - want)
    print(f"  worst {(err / (plain + 64 * 2.0 ** -17)).max():.2f} of its bound", flush=True)
    assert (err <= plain + 64 * 2.0 ** -17).all()


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", list(SCORES))
@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_a_row_does_not_see_may_hold_anything(d, scores, whole):
    """NaN and infinities in the K of a later token, and of another document in the same block, change no row before it (but for when its wave
    takes a new reference, hence the oracle and its bounds)."""
    cap, bias = SCORES[scores]
    flags = BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], dtype=torch.bfloat16, device=DEV)
    for lens, bs, plan in (([700, 90], 128, fcp.fcp_plan_blocks([700, 90], 128, 1, 2)),
                           ([50, 70, 8, 100], 256, fcp.fcp_plan_blocks_packed([50, 70, 8, 100], 256, 1, 0, None, [0, 0, 0, 0]))):
        run = Run(plan, 2, 1, d, bs, flags, backward=False, seed=14, softcap=cap, slopes=alibi(2) if bias else None)
        last = np.cumsum(lens) - 1
        for i, row in enumerate(last):
            run.k[row] = bad[i % 4]
        run.step()
        q, k, v, _ = (orc.bf16_to_f64(b) for b in run.bits)
        want = sorc.attention(q, k, v, *geometry(sorc.layout(lens, bs)), run.p.softcap, run.p.slopes)
        keep = np.setdiff1d(np.arange(run.p.t_q), last)
        for name, x in run.outputs().items():
            ref, bound = want[name]
            assert (np.abs(x - ref)[keep] <= bound[keep]).all(), name


@pytest.mark.parametrize("scores", ["bias", "both"])
def test_a_cache_of_more_than_2_31_elements(scores):
    """The last tokens of 270000, 64 KV heads: offsets into K and V pass 32 bits."""
    n, new, heads, d, bs = 270001, 33, 64, 128, 2048
    cap, _ = SCORES[scores]
    slopes = [2.0 ** -(4 + h % 16) for h in range(heads)]
    plan = fcp.fcp_plan_blocks_cut([n], [n - new], bs, 0, 16, [(0, -(-(n - new) // bs))])
    p = fcp.Problem(plan, heads, heads, d, bs, 0.0, BASE, softcap=cap, slopes=slopes)
    gen = torch.Generator(DEV).manual_seed(15)
    k, v = (torch.randn(n, heads, d, device=DEV, generator=gen, dtype=torch.bfloat16) for _ in range(2))
    q = torch.randn(new, heads, d, device=DEV, generator=gen, dtype=torch.bfloat16)
    assert k.numel() > 2 ** 31
    full = lambda *shape: torch.full(shape, float("nan"), device=DEV)
    o, lse, o_part, lse_part = full(new, heads, d), full(new, heads), full(p.n_slot_rows, heads, d), full(p.n_slot_rows, heads)
    size = fcp.fcp_workspace_bytes(p)
    ws = torch.zeros(size + 256, dtype=torch.uint8, device=DEV)
    ws_ptr = ws.data_ptr() + (-ws.data_ptr()) % 256
    fcp.fcp_queue_build(p, ws_ptr, size)
    fcp.fcp_block_attn_fwd_out(p, q, k, v, o_part, lse_part, o, lse, ws_ptr)
    fcp.fcp_merge_partials(p, o_part, lse_part, o, lse, ws_ptr)
    torch.cuda.synchronize()
    pos = np.arange(n)
    dist = np.abs(pos[n - new:, None] - pos[None])
    see = pos[None] <= pos[n - new:, None]
    for h in (0, 7, 63):
        x = [t[:, h:h + 1].double().cpu().numpy() for t in (q, k, v)]
        want = sorc.attention(*x, see, dist, cap, slopes[h:h + 1])
        for name, got in (("o", o), ("lse", lse)):
            ref, bound = want[name]
            assert (np.abs(got[:, h:h + 1].double().cpu().numpy() - ref) <= bound).all(), (h, name)


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
def test_two_graphs_share_a_workspace(whole):
    """Steps of two softcaps, which is read by every call, captured on one workspace and replayed in turn."""
    plan = fcp.fcp_plan_blocks([900, 300, 40], 128, 1, 2)
    flags = BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0)
    run = Run(plan, 4, 2, 64, 128, flags, seed=17, q_scale=2.0, softcap=20.0, slopes=alibi(4))
    eager, graphs = {}, {}
    side = torch.cuda.Stream()
    for cap in (20.0, 5.0, 100.0):
        run.p.scores.softcap = cap
        run.step()
        eager[cap] = run.outputs()
        graphs[cap] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[cap], stream=side):
            run.step(side)
    assert not np.array_equal(eager[20.0]["o"], eager[5.0]["o"])
    for cap in (5.0, 20.0, 100.0, 20.0, 5.0):
        graphs[cap].replay()
        for name, x in run.outputs().items():
            assert np.array_equal(x, eager[cap][name]), (cap, name)


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("spill", [0, fcp.FCP_FLAG_BWD_SPILL_DS], ids=["recompute", "spill"])
@pytest.mark.parametrize("lens,d", [([300, 40], 64), ([700, 260], 128)])
def test_layers_of_several_kinds_of_scores_take_turns_on_one_workspace(lens, d, spill, whole):
    """Plain and capped training steps on a workspace built with slopes leave the next biased step as it was, bit for bit."""
    plan = fcp.fcp_plan_blocks(lens, 128, 1, 2)
    flags = BASE | spill | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0)
    kinds = {"bias": dict(slopes=[0.5, 0.1]), "plain": {}, "cap": dict(softcap=20.0), "both": dict(softcap=5.0, slopes=[0.5, 0.1])}
    runs = {name: Run(plan, 2, 1, d, 128, flags, seed=1, **kw) for name, kw in kinds.items()}
    want = {}
    for name, run in runs.items():
        run.step()
        want[name] = run.outputs()
        run.ws_ptr = runs["bias"].ws_ptr
    for name in ("bias", "plain", "bias", "cap", "both", "plain", "cap", "bias", "both"):
        run = runs[name]
        for x in (run.o, run.lse, run.dq, run.dk, run.dv):
            x.fill_(float("nan"))
        run.step()
        for out, x in run.outputs().items():
            assert np.array_equal(x, want[name][out]), (name, out)


def test_a_workspace_is_known_for_as_long_as_nothing_is_built_over_it():
    """Many workspaces of one process (a layer each): what the first ones were built with still stands after the last."""
    plan = fcp.fcp_plan_blocks([300, 40], 128, 1, 2)
    bias = dict(slopes=[0.5, 0.1])
    plain, biased = (Run(plan, 2, 1, 64, 128, BASE, seed=1, **kw) for kw in ({}, bias))
    biased.step()
    want = biased.outputs()
    others = [Run(plan, 2, 1, 64, 128, BASE, seed=1, **kw) for kw in ({}, bias) * 50]
    with pytest.raises(fcp.FcpError) as e:                       # refused in front of any launch
        fcp.fcp_block_attn_fwd_out(biased.p, plain.q, plain.k, plain.v, plain.o_part, plain.lse_part, plain.o, plain.lse, plain.ws_ptr)
    assert e.value.code == -1 and "slopes" in str(e.value)
    plain.ws_ptr = biased.ws_ptr
    plain.step()
    biased.step()
    for name, x in biased.outputs().items():
        assert np.array_equal(x, want[name]), name
    # built over, from its start or from further in, the memory serves no slopes any more
    small = fcp.Problem(fcp.fcp_plan_blocks([16], 128, 1, 0), 1, 1, 64, 128, 0.0, BASE)
    assert fcp.fcp_workspace_bytes(small) <= fcp.fcp_workspace_bytes(biased.p) - 256
    for run, at in ((others[1], 0), (others[3], 256)):
        assert run.p.slopes is not None
        fcp.fcp_queue_build(small, run.ws_ptr + at, fcp.fcp_workspace_bytes(small))
        with pytest.raises(fcp.FcpError) as e:
            run.step()
        assert e.value.code == -1 and "slopes" in str(e.value)


def nearest_bound(run, see, dist):
    """What the oracle says of a row whose nearest key is far: its distance taken off all of them leaves O as it is and the LSE more by slope * that.
    The LSE's fp32 (this product, its sum and the change of base: seven roundings of half a step) is off by 2^-21 of its value."""
    near = np.where(see, dist, np.iinfo(np.int64).max).min(1)
    q, k, v, _ = (orc.bf16_to_f64(b) for b in run.bits)
    want = sorc.attention(q, k, v, see, dist - near[:, None], run.p.softcap, run.p.slopes)
    lse, el = want["lse"]
    lse = lse - near[:, None] * run.p.slopes.astype(np.float64)[None]
    return {"o": want["o"], "lse": (lse, el + 2.0 ** -21 * np.abs(lse))}


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", ["bias", "both", "wide"])
@pytest.mark.parametrize("far", [1003, 1000003, 20000001, 2 ** 30 + 1])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_whose_nearest_keys_are_far(d, far, scores, whole):
    """A share without the keys around its rows: rows far behind their keys, rows far before them, rows between two runs of keys and next to
    them, in blocks that follow each other and blocks that do not."""
    kv = [100, 128, 70, 128, 128, 33, 1, 128]
    kv_pos = [0, 100, 300, far + 3000, far + 3128, far + 3300, far + 90000, far + 3500]
    q_len, q_pos = [70, 130, 1, 40, 40], [far + 3000 - 200, 2 * far if far < 2 ** 30 else far + 200000, 3 * (far // 4), far + 3400, far + 3340]
    start = np.concatenate([[0], np.cumsum(kv)])
    q_start = np.concatenate([[0], np.cumsum(q_len)])
    see_blocks = [[0, 1, 2], [0, 1, 2, 6], [2, 0, 7, 3, 4, 5], [0, 6, 1], [7, 5]]
    pairs = [(b, j, 0, b) for b, js in enumerate(see_blocks) for j in js]
    slots, n = [], 0
    for b, js in enumerate(see_blocks):
        slots.append((b, n, len(js), q_start[b]))
        n += len(js)
    plan = dict(kv_blocks=[(0, i, start[i], n) for i, n in enumerate(kv)], q_blocks=[(0, 100 + b, q_start[b], n) for b, n in enumerate(q_len)],
                pairs=pairs, slots=slots, n_slot_rows=q_start[-1])
    slopes = [64.0, 8.0, 0.7, 2.0 ** -12]
    run = Run(plan, 4, 2, d, 130, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), backward=False, seed=21, q_scale=2.0, softcap=SCORES[scores][0], slopes=slopes,
              q_pos=q_pos, kv_pos=kv_pos)
    run.step()
    kp = np.concatenate([p + np.arange(n) for p, n in zip(kv_pos, kv)])
    qp = np.concatenate([p + np.arange(n) for p, n in zip(q_pos, q_len)])
    see = np.zeros((len(qp), len(kp)), dtype=bool)
    for b, js in enumerate(see_blocks):
        for j in js:
            see[q_start[b]:q_start[b + 1], start[j]:start[j + 1]] = True
    want = nearest_bound(run, see, np.abs(qp[:, None] - kp[None]))
    for name, x in run.outputs().items():
        ref, bound = want[name]
        assert np.isfinite(x).all(), name
        worst = (np.abs(x - ref) / bound).max()
        print(f"  {name}: worst {worst:.2f} of its bound", flush=True)
        assert worst <= 1.0, (name, worst)


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", ["bias", "both", "wide"])
def test_far_keys_get_no_gradient_from_rows_that_have_near_ones(scores, whole):
    """A share of keys that are all far, its backward given the LSE of rows whose near keys are elsewhere: P is 0 and so is every gradient."""
    plan = dict(kv_blocks=[(0, 0, 0, 100), (0, 1, 100, 128)], q_blocks=[(0, 9, 0, 90)], pairs=[(0, 0, 0, 0), (0, 1, 0, 0)], slots=[(0, 0, 2, 0)], n_slot_rows=90)
    run = Run(plan, 4, 2, 64, 128, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=22, softcap=SCORES[scores][0], slopes=[64.0, 8.0, 0.7, 0.01],
              q_pos=[2 ** 31 - 91], kv_pos=[0, 100])
    run.o.normal_()
    run.lse.normal_()
    fcp.fcp_block_attn_bwd(run.p, run.q, run.k, run.v, run.o, run.lse, run.d_o, run.dq, run.dk, run.dv, run.ws_ptr)
    for name, x in run.outputs().items():
        assert name in ("o", "lse") or not x.any(), name


FORMS = dict(SCORES, plain=(0.0, False))


def plan_of(geo):
    lens, bs, mask, cut, c, hq, hkv, d, owned = GEOMETRY[geo]
    plan = fcp.fcp_plan_blocks(lens, bs, int(mask == "causal"), c, owned) if cut is None else fcp.fcp_plan_blocks_cut(lens, cut, bs, int(mask == "prefix"), c, owned)
    return plan, (hq, hkv, d, bs), geometry(sorc.layout(lens, bs, cut=cut, owned=owned), mask, cut)


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("geo", [g for g in GEOMETRY if GEOMETRY[g][3] is not None])
def test_plain_scores_on_a_cut_plan(geo, whole):
    plan, shape, seen = plan_of(geo)
    for spill in (0, fcp.FCP_FLAG_BWD_SPILL_DS):
        run = Run(plan, *shape, BASE | spill | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), seed=31, q_scale=4.0)
        run.step()
        run.check(*seen)


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", FORMS)
@pytest.mark.parametrize("geo", ["ragged", "prefix_d128", "decode", "long_d128"])
def test_a_bf16_o_goes_out_and_into_the_backward(geo, scores, whole):
    """What inference hands out, and a training step that keeps no fp32 O: D is a sum over rounded values then, which the oracle's bound counts."""
    plan, shape, seen = plan_of(geo)
    cap, bias = FORMS[scores]
    for spill in (0, fcp.FCP_FLAG_BWD_SPILL_DS):
        flags = fcp.FCP_FLAG_DIRECT_SINGLE | fcp.FCP_FLAG_GRAD_BF16 | spill | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0)
        run = Run(plan, *shape, flags, seed=32, q_scale=3.0, softcap=cap, slopes=alibi(shape[0]) if bias else None)
        run.step()
        run.check(*seen)


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("scores", FORMS)
@pytest.mark.parametrize("o_flag", [0, fcp.FCP_FLAG_O_F32], ids=["bf16", "fp32"])
def test_bf16_partials(o_flag, scores, whole):
    """Each partial O is rounded once more: half a step of P|V|, which its slots share by their weights."""
    cap, bias = FORMS[scores]
    for geo in ("ragged_d128", "prefix", "decode_d128"):
        plan, shape, (see, dist) = plan_of(geo)
        flags = fcp.FCP_FLAG_DIRECT_SINGLE | fcp.FCP_FLAG_PART_BF16 | o_flag | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0)
        run = Run(plan, *shape, flags, backward=False, seed=33, q_scale=2.0, softcap=cap, slopes=alibi(shape[0]) if bias else None)
        run.o_part = torch.full_like(run.o_part, float("nan"), dtype=torch.bfloat16)
        run.step()
        q, k, v, _ = (orc.bf16_to_f64(b) for b in run.bits)
        want = sorc.attention(q, k, v, see, dist, cap, run.p.slopes, o_bf16=not o_flag)
        pv = sorc.attention(q, k, np.abs(v), see, dist, cap, run.p.slopes)["o"][0]
        got = run.outputs()
        # a partial is rounded with its errors of P in it (2 HALF P|V| at most), and the last rounding rounds this one's: 2 HALF^2 and HALF^2 more
        assert (np.abs(got["o"] - want["o"][0]) <= want["o"][1] + (sorc.HALF + 3 * sorc.HALF ** 2) * pv).all()
        assert (np.abs(got["lse"] - want["lse"][0]) <= want["lse"][1]).all()


@pytest.mark.parametrize("whole", [False, True], ids=["split", "whole"])
@pytest.mark.parametrize("cap", [20.0, 50.0, 60.3])
def test_values_up_to_the_stated_sum(cap, whole):
    """|v| of a row's keys summing up to 2^55, under scores at +softcap, at -softcap and in between."""
    lens, bs = [300, 65], 128
    plan = fcp.fcp_plan_blocks(lens, bs, 0, 1)
    run = Run(plan, 2, 1, 64, bs, BASE | (fcp.FCP_FLAG_WHOLE_ITEMS if whole else 0), backward=False, seed=23, softcap=cap)
    q, k, v = (workloads.bf16_to_f32(b) for b in run.bits[:3])
    k[..., 0] = 64.0
    q[0::3, :, 0], q[1::3, :, 0], q[2::3, :, 0] = -64.0, 64.0, 0.0
    v *= np.float32(2.0 ** 55 / np.abs(v).sum(0).max() * 0.99)
    for i, x in enumerate((q, k, v)):
        run.bits[i] = workloads.bf16_bits(x)
    run.q, run.k, run.v = (bits_to_dev(b) for b in run.bits[:3])
    run.step()
    run.check(*geometry(sorc.layout(lens, bs), "full"))
