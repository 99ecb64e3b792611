"""Operators around the block attention whose speed counts, as calls that a training or inference program makes.

Attention with modified scores.  For query row i and key j of one sequence, at positions i and j, and query head h:
    z = q_i . k_j / sqrt(d);   y = cap * tanh(z / cap) if cap else z;   s = y - slope_h * |i - j|
    P = softmax of s over the keys that row i sees;   O = P V;   LSE = ln sum exp(s)
and for training, from dO:  D = rowsum(dO o O);  dV = P^T dO;  dS = P o (dO V^T - D) o (1 - tanh^2(z / cap)) / sqrt(d);
dQ = dS K;  dK = dS^T Q.  A program plans a batch once and runs its tables for every layer: tables, queues, workspace and output
buffers belong to `prepare`.  Fields of a case:
  lens      "uniform" | "lognormal" (median `mid`, sigma 1), clipped to [lo, hi], until `tokens` are reached; "one": one sequence
  mask      "causal"; "full"; "prefix": the first tokens of a sequence (a share drawn between nothing and all of it) are seen
            by all of its rows, the others causally
  rows      "all" query rows; "new": the last `new` tokens of every sequence, what comes before is a cache; "zigzag": `owned` blocks
            of the sequence in pairs from both ends
  packed    neighbouring short sequences (documents) share a block
  cap, bias the cap (0: none); slopes 2^(-8 (h + 1) / heads) or none
  train, spill   forward and backward; the backward keeps dS in memory

Rotary positions with several axes.  Pair p of a head turns by pos[row][axis(p)] * freq(p); the gradient turns back.
  axes      position numbers of a token (3: time, height, width); the pairs are dealt to them by `split`: "runs" or "turns"
  inverse   False: Q and K out of a fused [rows, (hq + 2 hkv) d] projection into the attention's buffers;
            True: their gradients back into the fused layout
  far       highest position where a sequence may start
"""
import math

import numpy as np
import torch

own = False

_ATTN = dict(op="attn", batch=0, lens="lognormal", tokens=32768, lo=16, hi=32768, mid=2048, block=1024, coalesce=16,
             mask="causal", rows="all", new=0, owned=0, packed=False, hq=32, hkv=8, d=128, cap=0.0, bias=False, train=False,
             spill=False)
_ROPE = dict(op="rope", batch=0, rows=65536, hq=32, hkv=8, d=128, pairs=64, axes=3, split="runs", interleaved=False,
             theta=10000.0, far=32768, inverse=False, src32=False)


def _attn(name=None, **kw):
    c = dict(_ATTN, **kw)
    return dict(c, name=name) if name else c


def _rope(name=None, **kw):
    c = dict(_ROPE, **kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one step of a chat with few users and a small model: latency
        _attn("decode_small", lens="uniform", tokens=1500, lo=100, hi=700, block=128, coalesce=0, rows="new", new=1, hq=4, hkv=2,
              d=64, cap=30.0),
        # one step of a full batch: every cache is read once
        _attn("decode_batch", lens="uniform", tokens=196608, lo=500, hi=16000, rows="new", new=1, coalesce=4, cap=50.0),
        # evaluation / prefill over a packed batch, capped scores
        _attn("prefill_cap", cap=50.0),
        # the next 511 tokens of long prompts in chunked prefill, distance bias, odd group of heads
        _attn("chunk_bias", lens="uniform", tokens=65536, lo=2000, hi=20000, block=512, rows="new", new=511, hq=9, hkv=3, bias=True),
        # long-context prefill of one worker: zig-zag blocks of one sequence, partials to merge
        _attn("long_bias", lens="one", tokens=131072, block=2048, rows="zigzag", owned=12, hq=16, hkv=16, bias=True),
        # an encoder-decoder style batch: prompts (or images) seen as a whole, answers causal; small heads
        _attn("prefix_mix", lens="uniform", tokens=40000, lo=64, hi=4096, block=512, mask="prefix", hq=16, hkv=4, d=64, cap=20.0,
              bias=True),
        # the smallest training step
        _attn("train_tiny", lens="uniform", tokens=2000, lo=60, hi=400, block=128, coalesce=2, hq=4, hkv=2, d=64, cap=30.0,
              bias=True, train=True),
        # training step of one worker, capped scores, dS kept
        _attn("train_cap", cap=50.0, train=True, spill=True),
        # training on documents that share blocks, distance bias, nothing kept
        _attn("train_documents", lens="uniform", lo=16, hi=512, packed=True, hq=16, hkv=16, d=64, bias=True, train=True),
        # rotation of the tokens of one decoding step
        _rope("rope_decode", rows=33, far=1000000),
        # rotation in a training step: text, images and video frames
        _rope("rope_train"),
        # its gradient, from fp32 sums; part of each head rotated, neighbouring pairs
        _rope("rope_grad", rows=40001, hq=16, hkv=4, pairs=32, split="turns", interleaved=True, theta=500000.0, far=1000000,
              inverse=True, src32=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    batch = rng.randrange(1 << 20)
    hkv = rng.choice([1, 2, 3, 4, 8, 16])
    hq = hkv * rng.choice([1, 1, 2, 3, 4, 8])
    if rng.random() < 0.3:
        d = rng.choice([64, 128, 128, 256])
        inverse = rng.random() < 0.5
        return _rope(batch=batch, rows=min(_log_int(rng, 1, 65536), 2684354560 // ((hq + hkv) * d * 8)), hq=hq, hkv=hkv, d=d,
                     pairs=8 * rng.randrange(1, d // 16 + 1), axes=rng.choice([1, 2, 3, 3, 4]), split=rng.choice(["runs", "turns"]),
                     interleaved=rng.random() < 0.5, theta=rng.choice([10000.0, 500000.0, 1000000.0]), far=_log_int(rng, 1, 2000000),
                     inverse=inverse, src32=inverse and rng.random() < 0.5)
    while True:
        cap = rng.choice([0.0, rng.uniform(5, 60), math.exp(rng.uniform(math.log(5), math.log(200)))])
        bias = rng.random() < 0.5 or cap == 0.0
        train = rng.random() < 0.5
        mask = rng.choice(["causal", "causal", "causal", "prefix", "full"])
        c = _attn(batch=batch, hq=hq, hkv=hkv, d=rng.choice([64, 128, 128]), cap=cap, bias=bias, train=train, mask=mask,
                  spill=train and rng.random() < 0.4, block=rng.choice([64, 128, 256, 512, 777, 1024, 2048]),
                  coalesce=rng.choice([0, 1, 4, 16, 16]))
        kind = rng.choice(["uniform", "uniform", "lognormal", "lognormal", "one", "new", "documents"])
        if kind in ("uniform", "new"):
            hi = _log_int(rng, 2, 8192)
            c.update(lens="uniform", tokens=_log_int(rng, 500, 65536), lo=_log_int(rng, 1, hi - 1) if hi > 2 else 1, hi=hi)
            if kind == "new":
                c.update(rows="new", new=rng.choice([1, 1, 1, 2, 5, _log_int(rng, 1, 1000)]), mask="causal", train=False, spill=False)
        elif kind == "lognormal":
            c.update(tokens=_log_int(rng, 500, 65536), mid=_log_int(rng, 64, 8192))
        elif kind == "one":
            c.update(lens="one", tokens=_log_int(rng, 500, 131072), rows="zigzag", owned=2 * rng.randrange(1, 7), mask="causal", spill=False)
        else:
            c["block"] = rng.choice([512, 777, 1024, 2048])
            hi = _log_int(rng, 8, c["block"] - 1)
            c.update(lens="uniform", tokens=_log_int(rng, 500, 65536), lo=_log_int(rng, 1, hi - 1), hi=hi, packed=True,
                     mask=rng.choice(["causal", "full"]))
        g = _geometry(c)
        nnz = sum(_visible(c, s) for s in g)
        slots = 1 if c["coalesce"] == 0 else 1 + max(s[0] for s in g) // c["block"] // c["coalesce"]
        partials = sum(s[2] for s in g) * slots * c["hq"] * c["d"] * 4
        if work(c)["flops"] <= most and partials <= 6e9 and len(g) <= 600 and not (c["spill"] and 2 * nnz * c["hq"] > 12e9):
            return c


# ---------------------------------------------------------------- what a case is made of

def _lengths(c):
    if c["lens"] == "one":
        return [c["tokens"]]
    rng = np.random.default_rng([c["batch"], 0])
    out, total = [], 0
    while total < c["tokens"]:
        n = rng.integers(c["lo"], c["hi"]) if c["lens"] == "uniform" else np.clip(round(math.exp(rng.normal(math.log(c["mid"]), 1.0))), c["lo"], c["hi"])
        out.append(int(min(n, c["tokens"] - total)))
        total += out[-1]
    return out


def _geometry(c):
    """Per sequence: (tokens, first token cut at: prefix length or first new token, query rows, [(first row, rows), ..])."""
    rng = np.random.default_rng([c["batch"], 1])
    out = []
    for n in _lengths(c):
        cut, ranges = 0, [(0, n)]
        if c["mask"] == "prefix":
            cut = int(rng.integers(0, n + 1))
        if c["rows"] == "new":
            cut = max(0, n - c["new"])
            ranges = [(cut, n - cut)]
        elif c["rows"] == "zigzag":
            nb = -(-n // c["block"])
            low = np.sort(rng.choice(max(1, nb // 2), size=max(1, min(c["owned"] // 2, nb // 2)), replace=False))
            ranges = [(int(i) * c["block"], min(c["block"], n - int(i) * c["block"])) for i in np.unique(np.concatenate([low, nb - 1 - low]))]
        out.append((n, cut, sum(r for _, r in ranges), ranges))
    return out


def _visible(c, seq):
    """Score entries of one head of a sequence that are not masked."""
    n, cut, rows, ranges = seq
    if c["mask"] == "full":
        return rows * n
    entries = sum(r * a + r * (r + 1) // 2 for a, r in ranges)
    return entries + (cut * (cut - 1) // 2 if c["mask"] == "prefix" else 0)


def work(c):
    if c["op"] == "rope":
        n = c["rows"] * (c["hq"] + c["hkv"]) * c["d"]
        return {"bytes": n * (6 if c["src32"] else 4) + 4 * c["rows"] * c["axes"], "flops": 6 * c["rows"] * (c["hq"] + c["hkv"]) * c["pairs"]}
    g = _geometry(c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    q, kv, nnz = sum(s[2] for s in g) * hq, sum(s[0] for s in g) * hkv, sum(_visible(c, s) for s in g) * hq
    if not c["train"]:
        return {"bytes": 2 * d * (2 * q + 2 * kv) + 4 * q, "flops": 4 * d * nnz}
    return {"bytes": 2 * d * (4 * q + 4 * kv) + 4 * q, "flops": 14 * d * nnz}       # and dO in; dQ, dK, dV out


class _State:
    pass


def _units(lens, block):
    """Neighbouring sequences share a block while they fit: one unit number per sequence."""
    out, unit, left = [], -1, 0
    for n in lens:
        if n > left:
            unit, left = unit + 1, block
        left -= n
        out.append(unit)
    return out


def _slopes(c):
    return [2.0 ** (-8.0 * (h + 1) / c["hq"]) for h in range(c["hq"])] if c["bias"] else None


def _axis_of_pair(c):
    if c["split"] == "turns":
        return [p % c["axes"] for p in range(c["pairs"])]
    return [p * c["axes"] // c["pairs"] for p in range(c["pairs"])]


def _positions(c, rows):
    """Stretches of text (all axes count on together) and pictures (time stands still, height and width walk the grid)."""
    rng = np.random.default_rng([c["batch"], 2])
    out = np.empty((rows, c["axes"]), dtype=np.int32)
    row, at = 0, int(rng.integers(0, c["far"] + 1))
    while row < rows:
        n = int(min(rng.integers(1, 4096), rows - row))
        if c["axes"] > 1 and rng.random() < 0.5:
            w = int(rng.integers(1, 64))
            i = np.arange(n)
            out[row:row + n] = at
            out[row:row + n, -1] = at + i % w
            out[row:row + n, -2] = at + i // w
            at += max(w, n // w) + 1
        else:
            out[row:row + n] = (at + np.arange(n))[:, None]
            at += n
        row += n
        if rng.random() < 0.3:
            at = int(rng.integers(0, c["far"] + 1))           # the next sequence of the batch
    return out


def prepare(case, seed):
    c, s, dev = case, _State(), torch.device("cuda:0")
    s.case = c
    g = torch.Generator(device=dev).manual_seed(int(seed))

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(dtype)

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=dev)

    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["op"] == "rope":
        rows = c["rows"]
        s.pos = torch.from_numpy(_positions(c, rows)).to(dev)
        s.axis = _axis_of_pair(c)
        s.freq = [c["theta"] ** (-p / c["pairs"]) for p in range(c["pairs"])]
        fused = torch.zeros(rows, (hq + 2 * hkv) * d, dtype=torch.bfloat16, device=dev)
        dt = torch.float32 if c["src32"] else torch.bfloat16
        q, k = (fused[:, i * d:(i + n) * d].view(rows, n, d) for i, n in ((0, hq), (hq, hkv)))
        if c["inverse"]:
            s.src, s.dst = (normal(rows, hq, d, dtype=dt), normal(rows, hkv, d, dtype=dt)), (q, k)
        else:
            fused.copy_(normal(rows, (hq + 2 * hkv) * d))
            s.src, s.dst = (q, k), (empty(rows, hq, d), empty(rows, hkv, d))
        if own:
            import paper_2605_08524_amd as fcp
            s.rotary = fcp.Rotary(d, s.axis, s.freq, interleaved=c["interleaved"])
        return s

    s.geometry = _geometry(c)
    t_q, t_kv = sum(x[2] for x in s.geometry), sum(x[0] for x in s.geometry)
    # caps act on large scores: queries of twice the usual size
    s.q, s.k, s.v = normal(t_q, hq, d) * 2, normal(t_kv, hkv, d), normal(t_kv, hkv, d)
    if c["train"]:
        s.d_o = normal(t_q, hq, d)
    if not own:
        return s
    import paper_2605_08524_amd as fcp
    lens, bs = [x[0] for x in s.geometry], c["block"]
    if c["packed"]:
        plan = fcp.fcp_plan_blocks_packed(lens, bs, int(c["mask"] == "causal"), c["coalesce"], None, _units(lens, bs))
    elif c["mask"] == "prefix":
        plan = fcp.fcp_plan_blocks_cut(lens, [x[1] for x in s.geometry], bs, 1, c["coalesce"])
    elif c["rows"] == "new":
        # blocks are cut at the first new token; the blocks behind it are the query blocks
        owned = [(i, -(-cut // bs) + b) for i, (n, cut, rows, _) in enumerate(s.geometry) for b in range(-(-rows // bs))]
        plan = fcp.fcp_plan_blocks_cut(lens, [x[1] for x in s.geometry], bs, 0, c["coalesce"], owned)
    else:
        owned = [(0, a // bs) for a, _ in s.geometry[0][3]] if c["rows"] == "zigzag" else None
        plan = fcp.fcp_plan_blocks(lens, bs, int(c["mask"] == "causal"), c["coalesce"], owned)
    flags = fcp.FCP_FLAG_DIRECT_SINGLE
    if c["train"]:
        flags |= fcp.FCP_FLAG_GRAD_BF16 | (fcp.FCP_FLAG_BWD_SPILL_DS if c["spill"] else 0)
        s.dq, s.dk, s.dv = empty(t_q, hq, d), empty(t_kv, hkv, d), empty(t_kv, hkv, d)
    s.problem = fcp.Problem(plan, hq, hkv, d, bs, 0.0, flags, softcap=c["cap"], slopes=_slopes(c))
    s.o, s.lse = empty(t_q, hq, d), empty(t_q, hq, dtype=torch.float32)
    rows = max(1, s.problem.n_slot_rows)
    s.o_part, s.lse_part = empty(rows, hq, d, dtype=torch.float32), empty(rows, hq, dtype=torch.float32)
    n = fcp.fcp_workspace_bytes(s.problem)
    s.ws = torch.empty(n + 256, dtype=torch.uint8, device=dev)
    s.ws_ptr = s.ws.data_ptr() + (-s.ws.data_ptr()) % 256
    fcp.fcp_queue_build(s.problem, s.ws_ptr, n, torch.cuda.current_stream().cuda_stream)
    return s


# ---------------------------------------------------------------- a pass

def run(s):
    if not own:
        return _plain_rope(s) if s.case["op"] == "rope" else _plain_attn(s)
    import paper_2605_08524_amd as fcp
    stream = torch.cuda.current_stream().cuda_stream
    if s.case["op"] == "rope":
        fcp.fcp_rotary_apply(s.rotary, [(s.src[0], s.dst[0], s.pos), (s.src[1], s.dst[1], s.pos)], inverse=s.case["inverse"], stream=stream)
        return s.dst
    fcp.fcp_block_attn_fwd_out(s.problem, s.q, s.k, s.v, s.o_part, s.lse_part, s.o, s.lse, s.ws_ptr, stream)
    fcp.fcp_merge_partials(s.problem, s.o_part, s.lse_part, s.o, s.lse, s.ws_ptr, stream)
    if not s.case["train"]:
        return s.o, s.lse
    fcp.fcp_block_attn_bwd(s.problem, s.q, s.k, s.v, s.o, s.lse, s.d_o, s.dq, s.dk, s.dv, s.ws_ptr, stream)
    return s.o, s.lse, s.dq, s.dk, s.dv


def _plain_rope(s):
    c = s.case
    dev, pairs = s.pos.device, c["pairs"]
    # far positions: angles in 64 bits
    angle = s.pos.double()[:, s.axis] * torch.tensor(s.freq, dtype=torch.float64, device=dev)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin
    out = []
    for x in s.src:
        y = x.float().clone()
        if c["interleaved"]:
            a, b = y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]
        else:
            a, b = y[..., :pairs], y[..., pairs:2 * pairs]
        a2, b2 = a * cos - b * sin, a * sin + b * cos
        a.copy_(a2)
        b.copy_(b2)
        out.append(y.to(torch.bfloat16))
    return tuple(out)


def _plain_attn(s):
    """Sequence by sequence, at most `chunk` query rows at a time, in 32 bits."""
    c = s.case
    hq, hkv, d, cap = c["hq"], c["hkv"], c["d"], c["cap"]
    group, scale, dev = hq // hkv, 1.0 / math.sqrt(c["d"]), s.q.device
    slopes = torch.tensor(_slopes(c), device=dev).view(hkv, group, 1, 1) if c["bias"] else None
    out, out_lse = torch.empty_like(s.q), torch.empty(s.q.shape[:2], device=dev)
    if c["train"]:
        dq, dk, dv = torch.empty_like(s.q), torch.empty_like(s.k), torch.empty_like(s.v)
    at_q = at_kv = 0
    for n, cut, rows, ranges in s.geometry:
        k, v = (x[at_kv:at_kv + n].float().transpose(0, 1).contiguous() for x in (s.k, s.v))        # [hkv, n, d]
        if c["train"]:
            dk_seq, dv_seq = torch.zeros_like(k), torch.zeros_like(v)
        chunk = max(1, (1 << 28) // (hq * n))
        for first, count in ranges:
            for r0 in range(first, first + count, chunk):
                m = min(chunk, first + count - r0)
                at = at_q + r0 - first
                cols = n if c["mask"] == "full" else max(r0 + m, cut if c["mask"] == "prefix" else 0)
                kc, vc = k[:, :cols], v[:, :cols]
                q = s.q[at:at + m].float().view(m, hkv, group, d).permute(1, 2, 0, 3).reshape(hkv, group * m, d)
                z = torch.matmul(q, kc.transpose(1, 2).contiguous()).view(hkv, group, m, cols) * scale
                if cap:
                    t = torch.tanh(z * (1.0 / cap))
                    z = t * cap
                i, j = torch.arange(r0, r0 + m, device=dev)[:, None], torch.arange(cols, device=dev)[None]
                if c["bias"]:
                    z = z - slopes * (i - j).abs().float()
                if c["mask"] != "full":
                    hidden = j > i
                    if c["mask"] == "prefix":
                        hidden = hidden & (j >= cut)
                    z = z.masked_fill(hidden, float("-inf"))
                top = z.amax(-1, keepdim=True)
                p = torch.exp(z - top)
                total = p.sum(-1, keepdim=True)
                p = p / total
                o = torch.matmul(p.view(hkv, group * m, cols), vc).view(hkv, group, m, d)
                out[at:at + m] = o.permute(2, 0, 1, 3).reshape(m, hq, d).to(torch.bfloat16)
                out_lse[at:at + m] = (top + torch.log(total)).view(hq, m).t()
                if not c["train"]:
                    continue
                do = s.d_o[at:at + m].float().view(m, hkv, group, d).permute(1, 2, 0, 3).reshape(hkv, group * m, d)
                dv_seq[:, :cols] += torch.matmul(p.view(hkv, group * m, cols).transpose(1, 2).contiguous(), do)
                dp = torch.matmul(do, vc.transpose(1, 2).contiguous()).view(hkv, group, m, cols)
                delta = (do.view(hkv, group, m, d) * o).sum(-1, keepdim=True)
                ds = p * (dp - delta) * scale
                if cap:
                    ds = ds * (1 - t * t)
                ds = ds.view(hkv, group * m, cols)
                dk_seq[:, :cols] += torch.matmul(ds.transpose(1, 2).contiguous(), q)
                dq[at:at + m] = torch.matmul(ds, kc).view(hkv, group, m, d).permute(2, 0, 1, 3).reshape(m, hq, d).to(torch.bfloat16)
            at_q += count
        if c["train"]:
            dk[at_kv:at_kv + n] = dk_seq.transpose(0, 1).to(torch.bfloat16)
            dv[at_kv:at_kv + n] = dv_seq.transpose(0, 1).to(torch.bfloat16)
        at_kv += n
    return (out, out_lse, dq, dk, dv) if c["train"] else (out, out_lse)


# ---------------------------------------------------------------- the same from the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        # a pair as a complex number, turned by exp(+- i angle)
        pos = s.pos.cpu().numpy().astype(np.float64)
        turn = np.exp((-1j if c["inverse"] else 1j) * pos[:, s.axis] * np.asarray(s.freq))
        turn = torch.from_numpy(turn).to(s.pos.device)[:, None, :]
        out = []
        for x in s.src:
            y = x.double().clone()
            rot = y[..., :2 * c["pairs"]]
            pair = rot.unflatten(-1, (c["pairs"], 2)) if c["interleaved"] else rot.unflatten(-1, (2, c["pairs"])).transpose(-1, -2)
            w = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            y[..., :2 * c["pairs"]] = w.flatten(-2) if c["interleaved"] else w.transpose(-1, -2).flatten(-2)
            out.append(y)
        return tuple(out)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    group, dev = hq // hkv, s.q.device
    f64 = dict(dtype=torch.float64, device=dev)
    res = [torch.zeros(s.q.shape, **f64), torch.zeros(s.q.shape[:2], **f64)]
    if c["train"]:
        res += [torch.zeros(x.shape, **f64) for x in (s.q, s.k, s.v)]
    row_of, seq_first = [], 0
    for n, cut, rows, ranges in s.geometry:
        pos_q = np.concatenate([np.arange(a, a + r) for a, r in ranges]) if ranges else np.zeros(0, dtype=np.int64)
        row_of.append((seq_first, n, cut, pos_q))
        seq_first += n
    q_first = 0
    for kv0, n, cut, pos_q in row_of:
        pos_k = torch.arange(n, device=dev)
        step = max(1, (1 << 26) // max(1, n))
        for h in range(hq):
            kh, vh = s.k[kv0:kv0 + n, h // group].double(), s.v[kv0:kv0 + n, h // group].double()
            for r in range(0, len(pos_q), step):
                at = slice(q_first + r, q_first + min(r + step, len(pos_q)))
                pq = torch.from_numpy(pos_q[r:r + step]).to(dev)
                qh = s.q[at, h].double()
                score = qh @ kh.t().contiguous() / d ** 0.5
                if c["cap"]:
                    tanh = torch.tanh(score / c["cap"])
                    score = c["cap"] * tanh
                if c["bias"]:
                    score = score - _slopes(c)[h] * (pq[:, None] - pos_k[None]).abs().double()
                if c["mask"] != "full":
                    sees = pos_k[None] <= pq[:, None]
                    if c["mask"] == "prefix":
                        sees |= (pos_k < cut)[None]
                    score = torch.where(sees, score, torch.full((), -math.inf, **f64))
                lse = torch.logsumexp(score, 1)
                p = torch.exp(score - lse[:, None])
                o = p @ vh
                res[0][at, h], res[1][at, h] = o, lse
                if c["train"]:
                    doh = s.d_o[at, h].double()
                    res[4][kv0:kv0 + n, h // group] += p.t() @ doh
                    ds = p * (doh @ vh.t() - (doh * o).sum(1, keepdim=True)) / d ** 0.5
                    if c["cap"]:
                        ds = ds * (1 - tanh ** 2)
                    res[2][at, h] = ds @ kh
                    res[3][kv0:kv0 + n, h // group] += ds.t() @ qh
        q_first += len(pos_q)
    return tuple(res)
