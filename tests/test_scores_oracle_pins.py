"""The oracle of modified scores against closed forms, finite differences and torch's autograd in fp64."""
import numpy as np
import pytest
import torch

from oracle import fcp_oracle as orc
from oracle import fcp_scores_oracle as sorc


def _inputs(lens, hq, hkv, d, seed, **kw):
    rng = np.random.default_rng(seed)
    lay = sorc.layout(lens, 8, cut=kw.get("cut"), owned=kw.get("owned"))
    see = sorc.visible(*lay, mask=kw.get("mask", "causal"), cut=kw.get("cut"))
    dist = np.abs(lay[1][:, None] - lay[3][None])
    t_q, t_kv = see.shape
    return [rng.standard_normal((n, h, d)) for n, h in ((t_q, hq), (t_kv, hkv), (t_kv, hkv), (t_q, hq))], see, dist


def test_plain_scores_are_the_other_oracle():
    lens = [13, 1, 9]
    rng = np.random.default_rng(0)
    bits = [(rng.standard_normal((23, h, 64)).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16) for h in (4, 2, 2, 4)]
    q, k, v, do = (orc.bf16_to_f64(b) for b in bits)
    lay = sorc.layout(lens, 4)
    got = sorc.attention(q, k, v, sorc.visible(*lay), np.abs(lay[1][:, None] - lay[3][None]), d_o=do)
    o, lse = orc.worker_fwd(*bits[:3], lens, 4, 1)
    want = dict(zip(("dq", "dk", "dv"), orc.worker_bwd(*bits, lens, 4, 1)), o=o, lse=lse)
    for name, ref in want.items():
        assert np.allclose(got[name][0], ref, rtol=1e-10, atol=1e-12), name


@pytest.mark.parametrize("cap,slopes,mask", [(2.0, None, "causal"), (0.0, (0.5, 0.0), "full"), (1.5, (0.125, 2.0), "prefix")])
def test_against_autograd_and_differences(cap, slopes, mask):
    (q, k, v, do), see, dist = _inputs([11, 6], 2, 1, 8, 3, mask=mask, cut=[5, 0])
    got = sorc.attention(q, k, v, see, dist, cap, slopes, 0.7, do)
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))

    def loss(a, b, c):
        out = []
        for h in range(2):
            z = a[:, h] @ b[:, 0].T * 0.7
            s = cap * torch.tanh(z / cap) if cap else z
            if slopes is not None:
                s = s - slopes[h] * torch.tensor(dist)
            out.append(torch.softmax(s.masked_fill(~torch.tensor(see), -torch.inf), 1) @ c[:, 0])
        return (torch.stack(out, 1) * torch.tensor(do)).sum(), torch.stack(out, 1)
    val, o = loss(tq, tk, tv)
    val.backward()
    assert np.allclose(o.detach().numpy(), got["o"][0], atol=1e-12)
    for t, name in ((tq, "dq"), (tk, "dk"), (tv, "dv")):
        assert np.allclose(t.grad.numpy(), got[name][0], atol=1e-10), name
    rng = np.random.default_rng(1)
    for x, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        step = rng.standard_normal(x.shape)
        def at(e):
            arg = {"dq": q, "dk": k, "dv": v}
            arg[name] = x + e * step
            return (sorc.attention(arg["dq"], arg["dk"], arg["dv"], see, dist, cap, slopes, 0.7)["o"][0] * do).sum()
        assert abs((at(1e-5) - at(-1e-5)) / 2e-5 - (got[name][0] * step).sum()) < 1e-6, name


def test_closed_forms():
    (q, k, v, do), see, dist = _inputs([7], 2, 2, 8, 5)
    # equal keys: a steep slope leaves the own token, none the mean; a tiny cap makes every score alike
    o = sorc.attention(q, k, v, see, dist, 0.0, (1e4, 1e4))["o"][0]
    assert np.allclose(o, v)
    o, lse = (sorc.attention(q, k, v, see, dist, 2.0 ** -10)[n][0] for n in ("o", "lse"))
    assert np.allclose(lse, np.log(np.arange(1, 8))[:, None], atol=2e-3)
    assert np.allclose(o[6], v.mean(0), atol=5e-3)
    # a row that sees nothing
    see = see.copy()
    see[3] = False
    r = sorc.attention(q, k, v, see, dist, 3.0, (0.5, 0.5), d_o=do)
    assert np.all(r["o"][0][3] == 0) and np.all(np.isneginf(r["lse"][0][3])) and np.all(r["dq"][0][3] == 0)


@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_keys_without_weight_loosen_no_bound(cap):
    """Bounds of a row with far keys under a steep slope are those without them (to 1 %), and a bf16 half step of the outputs' terms or so."""
    (q, k, v, do), see, dist = _inputs([40], 2, 1, 16, 7)
    slopes = (40.0, 8.0)
    near = see & (dist < 8)
    far = dist + 1000 * (dist >= 8)
    a, b = (sorc.attention(q, k, v, s, far, cap, slopes, 0.25, do) for s in (near, see))
    for name in a:
        assert np.abs(a[name][0] - b[name][0]).max() < 1e-12, name
        assert (b[name][1] <= 1.01 * a[name][1]).all(), name
    half = sorc.HALF
    p_v = np.abs(v).repeat(2, 1)                                            # next to nothing but the own token is left
    assert (b["o"][1] <= 1.1 * half * 2 * p_v + 2e-3).all() and (b["lse"][1] <= 64 * 40.0 * 2.0 ** -21).all()
