"""Performance cases of the score-modified attention and of the rotary positions.

Attention cases run one rank's share (every ring step of the forward, then the backward) of packed
documents whose scores are capped by a tanh, biased by the distance of query and key, or seen through a
prefix mask.  Rotary cases turn the projections' outputs into the attention's operands and back:
queries rotated, keys rotated, concatenated and split from the values, in the order of the exchange's
send buffers.  A layer case runs both, as a training step of one attention layer does.

With `own` false a pass computes the operators in elementary 32-bit operations; with `own` true it calls
the library.

Layouts of an attention case (documents of lengths "docs", packed into one window):
  whole    every row against every row
  split    every query row; K/V arrive in `cp_r` consecutive chunks
  zigzag   rank `rank` of a ring of `cp_r`: two chunks of every document, cp_r steps
  tail     the last `rows` rows of the window against all of it
"""
import math

import torch

own = False

D_QK, D_V, D_NOPE, D_ROPE = 192, 128, 128, 64
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
# Most (query, key, head) triples of a case, masked ones too, that is, the largest listed case's.
MOST_TRIPLES = 8 * 16384 * 16384
DS_BUDGET_BYTES = 18 << 30


def _attn(name, docs, heads, kv_heads=0, layout="whole", cp_r=1, rank=0, rows=0, cap=0.0, bias=False, prefix="",
          q_scale=1.0, backward=True, planned=False):
    c = {"kind": "attn", "docs": ",".join(map(str, docs)), "heads": heads, "kv_heads": kv_heads, "layout": layout,
         "cp_r": cp_r, "rank": rank, "rows": rows, "cap": cap, "bias": bias, "prefix": prefix, "q_scale": q_scale,
         "backward": backward, "planned": planned}
    return dict(c, name=name) if name else c


def _rope(name, rows, heads, cp_u=1, pairs="32", pairing="interleaved", ladder="whole", first=0, grads="float32",
          backward=True):
    c = {"kind": "rope", "rows": rows, "heads": heads, "cp_u": cp_u, "pairs": pairs, "pairing": pairing,
         "ladder": ladder, "first": first, "grads": grads, "backward": backward}
    return dict(c, name=name) if name else c


def _layer(name, docs, heads, cap=0.0, bias=False, prefix="", pairs="32", pairing="interleaved", ladder="whole",
           q_scale=1.0):
    c = dict(_attn("", docs, heads, cap=cap, bias=bias, prefix=prefix, q_scale=q_scale), kind="layer", pairs=pairs,
             pairing=pairing, ladder=ladder)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest share: three packed documents, two K/V chunks, plans uploaded once and calls that
        # only launch, as in a recorded step; capped scores
        _attn("cap_tiny_2step", [64, 128, 320], 4, layout="split", cp_r=2, cap=50.0, planned=True),
        # a small micro-batch of three documents with a bias by distance
        _attn("bias_2k", [716, 285, 1047], 16, bias=True, planned=True),
        # short documents of lengths as they come, half of them prompts whose tokens see each other; 16
        # query heads on 2 K/V heads
        _attn("prefix_8k_ragged_gqa", [1304, 439, 937, 216, 1571, 675, 445, 1053, 640, 627], 16, 2,
              prefix="652,0,937,100,0,337,1,0,320,0"),
        # a micro-batch with one long document, capped and biased, sharper logits that reach the cap
        _attn("cap_bias_8k", [1304, 4096, 716, 1053, 1023], 8, cap=30.0, bias=True, q_scale=4.0),
        # one sequence over a ring of four steps, one head on the rank, of a length as it comes
        _attn("cap_ring16k_1head", [16411], 1, layout="zigzag", cp_r=4, rank=1, cap=50.0),
        # one new token of a long document: no gradient, bound by reading K and V
        _attn("token_64k", [65536], 16, layout="tail", rows=1, cap=50.0, bias=True, backward=False, planned=True),
        # the largest: one 16K document, prompt of a quarter, capped
        _attn("cap_prefix_16k", [16384], 8, cap=50.0, prefix="4096"),
        # rotary positions of one new token
        _rope("rope_token", 1, 16, first=65535, backward=False),
        # a video's axes (time, height, width), each with its own frequencies, pairs in halves of an axis'
        # columns that are no multiple of 16 bytes; odd rows, gradients received in 16 bits
        _rope("rope_video_1021", 1021, 64, cp_u=4, pairs="8,12,12", pairing="axis_halves", ladder="axis",
              grads="bfloat16"),
        # text and image tokens mixed: one ladder of frequencies over three axes
        _rope("rope_mixed_4k", 4096, 16, pairs="8,8,16", pairing="halves", first=120000),
        # the largest: a rank's 16K tokens of a 128-head model before the exchange over 8 ranks
        _rope("rope_text_16k", 16384, 128, cp_u=8, first=131072),
        # an attention layer between its projections, forward and backward
        _layer("layer_cap_8k", [1304, 1098, 439, 937, 1571, 716, 675, 445, 1007], 8, cap=50.0),
    ]


# ------------------------------------------------------------------ drawn cases

def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_docs(rng, total):
    """One document, or lengths of a packed window's mix (log-normal, median 1024)."""
    if total < 256 or rng.random() < 0.3:
        return [total]
    docs, left = [], total
    while left > 0:
        n = int(min(left, max(1, min(16384, rng.lognormvariate(math.log(1024), 0.9)))))
        docs.append(n)
        left -= n
    return docs


def _draw_scores(rng, docs):
    cap, bias, prefix = 0.0, False, ""
    while not (cap or bias or prefix):
        cap = rng.choice([0.0, 20.0, 30.0, 50.0])
        bias = rng.random() < 0.4
        if rng.random() < 0.4:
            prefix = ",".join(str(rng.choice([0, n, rng.randint(0, n)])) for n in docs)
    return {"cap": cap, "bias": bias, "prefix": prefix}


def _draw_attn(rng):
    layout = rng.choice(["whole", "whole", "split", "zigzag", "tail"])
    if layout == "tail":
        rows = _log_int(rng, 1, 64)
        total = _log_int(rng, 2 * rows, 131072)
        heads, kv = rng.choice([(1, 0), (4, 1), (8, 0), (16, 0), (16, 2)])
        docs = [total]
        backward = rng.random() < 0.3 and rows * total * heads < 1 << 26
        return _attn("", docs, heads, kv, layout, rows=rows, backward=backward, planned=rng.random() < 0.5,
                     q_scale=rng.choice([1.0, 4.0]), **_draw_scores(rng, docs))
    while True:
        total = _log_int(rng, 64, 16384)
        if rng.random() < 0.5:
            total = max(32, total // 32 * 32)
        heads, kv = rng.choice([(1, 0), (2, 0), (4, 0), (6, 3), (8, 0), (8, 2), (16, 0), (16, 2)])
        if total * total * heads <= MOST_TRIPLES:
            break
    cp_r, rank = 1, 0
    if layout != "whole":
        cp_r = rng.choice([2, 4])
        rank = rng.randrange(cp_r) if layout == "zigzag" else 0
    if layout == "zigzag":
        cut = rng.randint(1, total - 1)
        docs = [total] if rng.random() < 0.5 else [cut, total - cut]
    else:
        docs = _draw_docs(rng, total)
    return _attn("", docs, heads, kv, layout, cp_r, rank, planned=rng.random() < 0.4, backward=rng.random() < 0.8,
                 q_scale=rng.choice([1.0, 1.0, 4.0]), **_draw_scores(rng, docs))


def _draw_rope_kind(rng):
    pairing = rng.choice(["interleaved", "halves", "axis_halves"])
    ladder = rng.choice(["whole", "axis"])
    n = rng.choice([1, 1, 2, 3])
    if n == 1:
        pairs = [32]
    else:
        cuts = sorted(rng.sample(range(1, 32), n - 1))
        pairs = [b - a for a, b in zip([0] + cuts, cuts + [32])]
    return {"pairs": ",".join(map(str, pairs)), "pairing": pairing, "ladder": ladder}


def draw(rng):
    kind = rng.choice(["attn"] * 5 + ["rope"] * 3 + ["layer"])
    if kind == "attn":
        return _draw_attn(rng)
    if kind == "rope":
        heads = rng.choice([1, 4, 8, 16, 64, 128])
        return _rope("", _log_int(rng, 1, (2 << 20) // heads), heads,
                     cp_u=rng.choice([n for n in (1, 2, 4, 8) if n <= heads]), first=rng.choice([0, 1000, 250000]),
                     grads=rng.choice(["float32", "float32", "bfloat16"]), backward=rng.random() < 0.8,
                     **_draw_rope_kind(rng))
    docs = _draw_docs(rng, _log_int(rng, 32, 8192))
    return _layer("", docs, rng.choice([1, 2, 4, 8, 16]), q_scale=rng.choice([1.0, 4.0]), **_draw_scores(rng, docs),
                  **_draw_rope_kind(rng))


# ------------------------------------------------------------------ what a case is

def _ints(text):
    return [int(n) for n in text.split(",")] if text else []


def _geometry(c):
    """Document boundaries, the rank's query segments and the K/V segments of every ring step."""
    lengths = _ints(c["docs"])
    cu = [0]
    for n in lengths:
        cu.append(cu[-1] + n)
    total, cp, r = cu[-1], c["cp_r"], c["rank"]
    if c["layout"] == "whole":
        return cu, [(0, total)], [[(0, total)]]
    if c["layout"] == "tail":
        return cu, [(total - c["rows"], c["rows"])], [[(0, total)]]
    if c["layout"] == "split":
        edge = [j * total // cp for j in range(cp + 1)]
        return cu, [(0, total)], [[(edge[j], edge[j + 1] - edge[j])] for j in range(cp)]

    def rows_of(x):
        out = []
        for base, n in zip(cu, lengths):
            edge = [j * n // (2 * cp) for j in range(2 * cp + 1)]
            for j in (x, 2 * cp - 1 - x):
                out.append((base + edge[j], edge[j + 1] - edge[j]))
        return out
    return cu, rows_of(r), [rows_of((r - i) % cp) for i in range(cp)]


def _pairs(c):
    """Visible (query, key) pairs of one head."""
    cu, q_segs, steps = _geometry(c)
    prefix = _ints(c["prefix"]) or [0] * (len(cu) - 1)
    n = 0
    for d0, d1, px in zip(cu[:-1], cu[1:], prefix):
        for qs, qn in q_segs:
            qa, qb = max(qs, d0), min(qs + qn, d1)
            for step in steps:
                for ks, kn in step:
                    ka, kb = max(ks, d0), min(ks + kn, d1)
                    if qb <= qa or kb <= ka:
                        continue
                    # sum over p in [qa, qb) of the keys in [ka, min(kb, max(p + 1, d0 + px)))
                    e = d0 + px  # every row sees the keys before e; rows from e on see up to themselves
                    low = max(0, min(kb, e) - ka)
                    n += max(0, min(qb, e) - qa) * low
                    a = max(qa, e)
                    if a < qb:
                        first, last = a + 1 - ka, qb - ka  # p + 1 - ka for the rows left
                        width = kb - ka
                        n += max(0, last - max(first, width) + 1) * width
                        lo, hi = max(first, 1), min(last, width - 1)
                        if hi >= lo:
                            n += (lo + hi) * (hi - lo + 1) // 2
    return n


def _attn_work(c):
    _, q_segs, steps = _geometry(c)
    H, Hk = c["heads"], c["kv_heads"] or c["heads"]
    nq, nk = sum(n for _, n in q_segs), sum(n for s in steps for _, n in s)
    n = _pairs(c) * H
    # forward: Q, K, V read; O and LSE written.  Backward: dO read; dQ, dK, dV written
    b = nq * H * (D_QK * 2 + D_V * 2 + 4) + nk * Hk * (D_QK + D_V) * 2
    f = 640.0 * n
    if c["backward"]:
        b += nq * H * (D_V + D_QK) * 2 + nk * Hk * (D_QK + D_V) * 2
        f += 1664.0 * n
    return b, f


def _rope_work(rows, heads, grads, backward, axes):
    # forward: q, kv and k_pe read; q, k, v written.  Backward: dq, dk, dv read; d_q, d_kv, d_k_pe written
    n = rows * heads
    b = n * (2 * D_QK + D_NOPE + D_V + D_QK + D_V) * 2 + rows * (D_ROPE * 2 + 4 * axes)
    if backward:
        b += n * (2 * D_QK + D_V) * grads + n * (D_QK + D_NOPE + D_V) * 2 + rows * D_ROPE * 2
    # two products and a sum per rotated value of q, per rotated key value before it is shared
    f = 3.0 * (n + rows) * D_ROPE * (2 if backward else 1) + (n * D_ROPE if backward else 0)
    return b, f


def work(c):
    if c["kind"] == "attn":
        b, f = _attn_work(c)
    elif c["kind"] == "rope":
        b, f = _rope_work(c["rows"], c["heads"], 4 if c["grads"] == "float32" else 2, c["backward"],
                          len(_ints(c["pairs"])))
    else:
        # the operands of the attention and their gradients stay inside the layer
        b, f = _attn_work(c)
        rows = sum(_ints(c["docs"]))
        b2, f2 = _rope_work(rows, c["heads"], 4, True, len(_ints(c["pairs"])))
        b, f = rows * (c["heads"] * 2 * (D_QK + D_NOPE + D_V + D_V) * 2 + 4 * D_ROPE), f + f2
    return {"bytes": float(b), "flops": f}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, shape, scale=1.0, dtype=BF16):
    """N(0, scale^2), drawn and scaled in 32 bits and rounded once."""
    t = torch.randn(shape, generator=g, device="cuda", dtype=F32)
    if scale != 1.0:
        t *= scale
    return t.to(dtype)


def _score_inputs(c):
    """What describes a case's scores: the heads' slopes (a geometric ladder from 2^(-8/H) to 2^-8) and
    every document's prefix."""
    H = c["heads"]
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=F32, device="cuda") if c["bias"] else None
    return slopes, _ints(c["prefix"]) or None


def _attn_inputs(c, seed):
    """Projections of normalised activations: q and k near N(0, 1) (logits of unit variance, or 16 where
    q_scale is 4), v ~ N(0, 1)/sqrt(128), dO ~ N(0, 1)."""
    _, q_segs, steps = _geometry(c)
    H, Hk = c["heads"], c["kv_heads"] or c["heads"]
    g = _gen(seed)
    nq = sum(n for _, n in q_segs)
    q = _randn(g, (nq, H, D_QK), c["q_scale"])
    kv = []
    for s in steps:
        nk = sum(n for _, n in s)
        kv.append((_randn(g, (nk, Hk, D_QK)), _randn(g, (nk, Hk, D_V), 1 / math.sqrt(D_V))))
    d_o = _randn(g, (nq, H, D_V)) if c["backward"] else None
    return q, kv, d_o


def _rope_positions(n_axes, rows, first, seed):
    """Text: consecutive positions from `first` on.  Several axes: the frames of a video of 16 x 24 tokens
    each, from frame `first`, row by row."""
    i = torch.arange(rows, device="cuda", dtype=torch.int64)
    if n_axes == 1:
        p = [i + first]
    elif n_axes == 2:
        p = [i // 24, i % 24 + first]
    else:
        p = [first + i // 384, i // 24 % 16, i % 24]
    return (torch.stack(p) + seed % 7).to(torch.int32)


def _rope_inputs(c, seed):
    g = _gen(seed)
    n, H, u = c["rows"], c["heads"], c["cp_u"]
    x = {"q": _randn(g, (n, H, D_QK)), "kv": _randn(g, (n, H, D_NOPE + D_V)), "k_pe": _randn(g, (n, D_ROPE))}
    x["pos"] = _rope_positions(len(_ints(c["pairs"])), n, c["first"], seed)
    if c["backward"]:
        t = F32 if c["grads"] == "float32" else BF16
        for name, d in (("dq", D_QK), ("dk", D_QK), ("dv", D_V)):
            x[name] = _randn(g, (u, n, H // u, d), dtype=t)
    return x


def _layer_inputs(c, seed):
    g = _gen(seed)
    n, H = sum(_ints(c["docs"])), c["heads"]
    x = {"q": _randn(g, (n, H, D_QK), c["q_scale"]), "k_pe": _randn(g, (n, D_ROPE)), "d_o": _randn(g, (n, H, D_V))}
    kv = torch.randn((n, H, D_NOPE + D_V), generator=g, device="cuda", dtype=F32)
    kv[..., D_NOPE:] *= 1 / math.sqrt(D_V)
    x["kv"] = kv.to(BF16)
    axes = len(_ints(c["pairs"]))
    # every document starts anew
    x["pos"] = torch.cat([_rope_positions(axes, m, 0, seed) for m in _ints(c["docs"])], 1)
    return x


def _row_positions(segs):
    return torch.cat([torch.arange(a, a + n, device="cuda") for a, n in segs])


def _window(c):
    """Positions, document starts, document numbers and prefix ends of the rank's rows."""
    cu, q_segs, steps = _geometry(c)
    edge = torch.tensor(cu, device="cuda")
    prefix = torch.tensor(_ints(c["prefix"]) or [0] * (len(cu) - 1), device="cuda")
    qp, kp = _row_positions(q_segs), torch.cat([_row_positions(s) for s in steps])
    qd, kd = (torch.searchsorted(edge, p, right=True) - 1 for p in (qp, kp))
    return {"qp": qp, "kp": kp, "qd": qd, "kd": kd, "pe": (edge[:-1] + prefix)[qd]}


def _pair_columns(c):
    """The two columns, the axis and the frequency (radians per position) of every rotated pair."""
    pairs = _ints(c["pairs"])
    n = sum(pairs)
    a, b, axis, freq, j0 = [], [], [], [], 0
    for x, m in enumerate(pairs):
        for j in range(j0, j0 + m):
            cols = {"interleaved": (2 * j, 2 * j + 1), "halves": (j, n + j),
                    "axis_halves": (j0 + j, j0 + j + m)}[c["pairing"]]
            a.append(cols[0])
            b.append(cols[1])
            axis.append(x)
            freq.append(10000.0 ** -((j - j0) / m if c["ladder"] == "axis" else j / n))
        j0 += m
    return a, b, axis, freq


# ------------------------------------------------------------------ a user's program

def prepare(c, seed):
    s = {"case": dict(c)}
    if c["kind"] == "attn":
        q, kv, d_o = _attn_inputs(c, seed)
        s.update(q=q, kv=kv, d_o=d_o)
    elif c["kind"] == "rope":
        s.update(_rope_inputs(c, seed))
    else:
        s.update(_layer_inputs(c, seed))
    if c["kind"] != "rope":
        s["slopes"], s["prefix"] = _score_inputs(c)
    if c["kind"] != "attn":
        a, b, axis, freq = _pair_columns(c)
        s["a"], s["b"], s["axis"] = (torch.tensor(v, device="cuda") for v in (a, b, axis))
        s["freq"] = torch.tensor(freq, dtype=F64, device="cuda")
    if own:
        _prepare_own(c, s)
    elif c["kind"] != "rope":
        s["window"] = _window(c)
    return s


def _prepare_own(c, s):
    """Plans, workspaces, accumulators and outputs that a program keeps."""
    from paper_2609_34318_amd import hydra, ring
    empty = lambda shape, t=BF16: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    if c["kind"] != "rope":
        cu, q_segs, steps = _geometry(c)
        H, Hk = c["heads"], c["kv_heads"] or c["heads"]
        scores = hydra.Scores(softcap=c["cap"], slopes=s["slopes"], prefix=s["prefix"])
        store = c["backward"] and not c["planned"]
        share = ring.make_share(cu, H, q_segs, steps, n_kv_heads=Hk, graph_ready=c["planned"], scores=scores,
                                ds_budget_bytes=DS_BUDGET_BYTES if store else 0)
        if c["planned"]:
            ring.plan(share)
        s["share"] = share
        if c["backward"]:
            s["dq"] = empty((share.nq, H, D_QK), F32)
            s["dkv"] = [(empty((p.nk, Hk, D_QK), F32), empty((p.nk, Hk, D_V), F32)) for p in share.problems]
    if c["kind"] != "attn":
        n, H, u = s["q"].shape[0], c["heads"], c.get("cp_u", 1)
        s["rope"] = hydra.Rope(pairs=_ints(c["pairs"]), pairing=c["pairing"], ladder=c["ladder"], base=10000.0)
        s["q_out"], s["k_out"] = (empty((u, n, H // u, D_QK)) for _ in range(2))
        s["v_out"] = empty((u, n, H // u, D_V))
        if c["backward"]:
            s["d_q"], s["d_kv"], s["d_k_pe"] = (torch.empty_like(s[x]) for x in ("q", "kv", "k_pe"))


def _own_share(c, s, q, kv, d_o):
    from paper_2609_34318_amd import ring
    _, lse, o16 = ring.forward(s["share"], q, kv, planned=c["planned"])
    if d_o is not None:
        s["dq"].zero_()
        for dk, dv in s["dkv"]:
            dk.zero_()
            dv.zero_()
        ring.backward(s["share"], q, kv, d_o, s["dq"], s["dkv"], planned=c["planned"])
    return o16, lse


def _run_own(c, s):
    from paper_2609_34318_amd import hydra
    if c["kind"] == "attn":
        o, lse = _own_share(c, s, s["q"], s["kv"], s["d_o"])
        out = {"o": o, "lse": lse}
        if c["backward"]:
            out.update(dq=s["dq"].to(BF16), dk=[k.to(BF16) for k, _ in s["dkv"]], dv=[v.to(BF16) for _, v in s["dkv"]])
        return out
    u = c.get("cp_u", 1)
    hydra.rope_q(s["rope"], s["q"], s["pos"], s["q_out"], cp_u=u)
    hydra.rope_kv(s["rope"], s["kv"], s["k_pe"], s["pos"], s["k_out"], s["v_out"], cp_u=u)
    if c["kind"] == "rope":
        out = {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
        grads = [s[x] for x in ("dq", "dk", "dv")] if c["backward"] else None
    else:
        o, lse = _own_share(c, s, s["q_out"][0], [(s["k_out"][0], s["v_out"][0])], s["d_o"])
        out = {"o": o, "lse": lse}
        grads = [s["dq"], *s["dkv"][0]]
    if grads:
        hydra.rope_q_bwd(s["rope"], grads[0], s["pos"], s["d_q"], cp_u=u)
        hydra.rope_kv_bwd(s["rope"], grads[1], grads[2], s["pos"], s["d_kv"], s["d_k_pe"], cp_u=u)
        out.update(d_q=s["d_q"], d_kv=s["d_kv"], d_k_pe=s["d_k_pe"])
    return out


# ------------------------------------------------------------------ the plain form

def _plain_attention(c, s, q, k, v, d_o):
    """O, LSE, dQ, dK, dV in 32 bits from [rows, heads, columns] operands in 32 bits."""
    w = s["window"]
    H, Hk = c["heads"], c["kv_heads"] or c["heads"]
    heads = lambda t: t.reshape(t.shape[0], Hk, -1, t.shape[-1]).permute(1, 2, 0, 3).contiguous()  # noqa: E731
    rows = lambda t: t.permute(2, 0, 1, 3).reshape(t.shape[2], -1, t.shape[3])  # noqa: E731
    q, k, v = heads(q), heads(k), heads(v)
    scale = 1 / math.sqrt(D_QK)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    if c["cap"]:
        x = torch.tanh(x / c["cap"])
        f = 1 - x * x if d_o is not None else None
        x = x * c["cap"]
    if c["bias"]:
        far = (w["qp"][:, None] - w["kp"][None, :]).abs().to(F32)
        x = x - s["slopes"].reshape(Hk, -1, 1, 1) * far
    sees = (w["qd"][:, None] == w["kd"][None, :]) & ((w["kp"][None, :] <= w["qp"][:, None]) | (w["kp"][None, :] < w["pe"][:, None]))
    x = torch.where(sees, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).reshape(H, -1)
    p = x / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, v)
    if d_o is None:
        return rows(o), lse, None, None, None
    d_o = heads(d_o)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), d_o).sum(1, keepdim=True)
    ds = p * (torch.matmul(d_o, v.transpose(-1, -2).contiguous()) - (d_o * o).sum(-1, keepdim=True)) * scale
    if c["cap"]:
        ds = ds * f
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q).sum(1, keepdim=True)
    return rows(o), lse, rows(dq), rows(dk), rows(dv)


def _turn(s, x, back=False):
    """Columns of x [..., rows, heads or 1, 64] (32 bits) rotated by their rows' angles."""
    angle = s["pos"].to(F64)[s["axis"]].t() * s["freq"]  # 64 bits: far positions
    cos, sin = (t.to(F32)[:, None] for t in (torch.cos(angle), torch.sin(-angle if back else angle)))
    a, b = x[..., s["a"]], x[..., s["b"]]
    y = torch.empty_like(x)
    y[..., s["a"]] = a * cos - b * sin
    y[..., s["b"]] = b * cos + a * sin
    return y


def _send(x, u):
    """[rows, heads, d] -> [u, rows, heads / u, d]"""
    return x.reshape(x.shape[0], u, -1, x.shape[-1]).transpose(0, 1).contiguous()


def _received(x):
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[-1])


def _plain_rope(s, q, kv, k_pe):
    q = torch.cat([q[..., :D_NOPE], _turn(s, q[..., D_NOPE:])], -1)
    pe = _turn(s, k_pe[:, None])
    k = torch.cat([kv[..., :D_NOPE], pe.expand(-1, kv.shape[1], -1)], -1)
    return q, k, kv[..., D_NOPE:]


def _plain_rope_bwd(s, dq, dk, dv):
    d_q = torch.cat([dq[..., :D_NOPE], _turn(s, dq[..., D_NOPE:], True)], -1)
    d_k_pe = _turn(s, dk[..., D_NOPE:].sum(1, keepdim=True), True)[:, 0]
    return d_q, torch.cat([dk[..., :D_NOPE], dv], -1), d_k_pe


def _run_plain(c, s):
    if c["kind"] == "attn":
        k, v = (torch.cat([t[i] for t in s["kv"]]).to(F32) for i in (0, 1))
        d_o = s["d_o"].to(F32) if c["backward"] else None
        o, lse, dq, dk, dv = _plain_attention(c, s, s["q"].to(F32), k, v, d_o)
        out = {"o": o.to(BF16), "lse": lse}
        if c["backward"]:
            sizes = [t[0].shape[0] for t in s["kv"]]
            out.update(dq=dq.to(BF16), dk=list(dk.to(BF16).split(sizes)), dv=list(dv.to(BF16).split(sizes)))
        return out
    q, k, v = _plain_rope(s, s["q"].to(F32), s["kv"].to(F32), s["k_pe"].to(F32))
    if c["kind"] == "rope":
        u = c["cp_u"]
        out = {n: _send(x.to(BF16), u) for n, x in (("q", q), ("k", k), ("v", v))}
        if not c["backward"]:
            return out
        grads = [_received(s[x]).to(F32) for x in ("dq", "dk", "dv")]
    else:
        # the operands of the attention are 16-bit tensors, as its callers have them
        o, lse, *grads = _plain_attention(c, s, q.to(BF16).to(F32), k.to(BF16).to(F32), v, s["d_o"].to(F32))
        out = {"o": o.to(BF16), "lse": lse}
    d_q, d_kv, d_k_pe = _plain_rope_bwd(s, *grads)
    out.update(d_q=d_q.to(BF16), d_kv=d_kv.to(BF16), d_k_pe=d_k_pe.to(BF16))
    return out


def run(s):
    return _run_own(s["case"], s) if own else _run_plain(s["case"], s)


# ------------------------------------------------------------------ 64-bit results

def _exact_attention(c, q, k, v, d_o):
    """One head and one block of query rows at a time, each row's softmax over the keys it may see."""
    cu, q_segs, steps = _geometry(c)
    slopes, prefix = _score_inputs(c)
    H, Hk = c["heads"], c["kv_heads"] or c["heads"]
    nq, nk = q.shape[0], k.shape[0]
    qp = _row_positions(q_segs)
    kp = torch.cat([_row_positions(st) for st in steps])
    # the interval of positions that a row sees
    starts = torch.zeros_like(qp)
    ends = qp + 1
    for i, (a, b) in enumerate(zip(cu[:-1], cu[1:])):
        inside = (qp >= a) & (qp < b)
        starts = torch.where(inside, a, starts)
        ends = torch.where(inside, ends.clamp(min=a + (prefix[i] if prefix else 0)), ends)
    O = torch.zeros((nq, H, D_V), dtype=F64, device="cuda")
    L = torch.full((H, nq), -math.inf, dtype=F64, device="cuda")
    dq = torch.zeros((nq, H, D_QK), dtype=F64, device="cuda")
    dk = torch.zeros((nk, Hk, D_QK), dtype=F64, device="cuda")
    dv = torch.zeros((nk, Hk, D_V), dtype=F64, device="cuda")
    scale = 1 / math.sqrt(D_QK)
    for b0 in range(0, nq, 2048):
        rows = slice(b0, min(nq, b0 + 2048))
        hidden = (kp[None] < starts[rows, None]) | (kp[None] >= ends[rows, None])
        far = (qp[rows, None] - kp[None]).abs().to(F64) if c["bias"] else None
        for h in range(H):
            g = h // (H // Hk)
            qh, kh, vh = q[rows, h].to(F64), k[:, g].to(F64), v[:, g].to(F64)
            z = qh @ kh.t() * scale
            if c["cap"]:
                th = torch.tanh(z / c["cap"])
                z = c["cap"] * th
            if c["bias"]:
                z = z - float(slopes[h]) * far
            z.masked_fill_(hidden, -math.inf)
            lse = torch.logsumexp(z, 1)
            P = torch.exp(z - lse.masked_fill(lse == -math.inf, 0.0)[:, None])
            oh = P @ vh
            O[rows, h], L[h, rows] = oh, lse
            if d_o is None:
                continue
            do = d_o[rows, h].to(F64)
            dz = P * (do @ vh.t() - (do * oh).sum(1, keepdim=True))
            if c["cap"]:
                dz = dz * (1 - th ** 2)
            dz = dz * scale
            dq[rows, h] = dz @ kh
            dk[:, g] += dz.t() @ qh
            dv[:, g] += P.t() @ do
    return O, L, dq, dk, dv


def _exact_turn(c, pos, x, sign):
    """The pairs as complex numbers times e^(i sign angle)."""
    a, b, axis, freq = _pair_columns(c)
    angle = torch.stack([pos[axis[j]].to(F64) * freq[j] for j in range(len(a))], 1)
    z = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * torch.polar(torch.ones_like(angle), sign * angle)[:, None]
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(c, seed):
    if c["kind"] == "attn":
        q, kv, d_o = _attn_inputs(c, seed)
        O, L, dq, dk, dv = _exact_attention(c, q, torch.cat([k for k, _ in kv]), torch.cat([v for _, v in kv]), d_o)
        out = {"o": O, "lse": L}
        if c["backward"]:
            sizes = [k.shape[0] for k, _ in kv]
            out.update(dq=dq, dk=list(dk.split(sizes)), dv=list(dv.split(sizes)))
        return out
    x = _rope_inputs(c, seed) if c["kind"] == "rope" else _layer_inputs(c, seed)
    q, kv, pe = x["q"].to(F64), x["kv"].to(F64), x["k_pe"].to(F64)[:, None]
    q[..., D_NOPE:] = _exact_turn(c, x["pos"], q[..., D_NOPE:], 1)
    pe = _exact_turn(c, x["pos"], pe, 1)
    k = torch.cat([kv[..., :D_NOPE], pe.expand(-1, kv.shape[1], -1)], -1)
    v = kv[..., D_NOPE:]
    u = c.get("cp_u", 1)
    if c["kind"] == "rope":
        split = lambda t: torch.stack(t.chunk(u, 1))  # noqa: E731
        out = {"q": split(q), "k": split(k), "v": split(v)}
        if not c["backward"]:
            return out
        dq, dk, dv = (torch.cat(list(x[n].to(F64)), 1) for n in ("dq", "dk", "dv"))
    else:
        O, L, dq, dk, dv = _exact_attention(c, q.to(BF16), k.to(BF16), v, x["d_o"])
        out = {"o": O, "lse": L}
    dq[..., D_NOPE:] = _exact_turn(c, x["pos"], dq[..., D_NOPE:], -1)
    d_pe = _exact_turn(c, x["pos"], dk[..., D_NOPE:].sum(1, keepdim=True), -1)[:, 0]
    out.update(d_q=dq, d_kv=torch.cat([dk[..., :D_NOPE], dv], -1), d_k_pe=d_pe)
    return out
