"""The attention branch's operators for training and streaming, as a user's program calls them.

Three operators that belong together, and their gradients:

* rotary positions with several axes (latent frame, row, column) of the query
  and key heads, from the token grid or from positions of the user's own, and
  the same rotation taken back, which is its gradient;
* attention that keeps the logarithm of each row's sum, over packed or padded
  sequences, with key heads shared by several query heads, and with frames
  that see only the frames of a window (causal in frames, or local in time);
* its gradient, which recomputes the probabilities from that logarithm.

Head counts, head dims and token counts are the ones of the shapes this
repository is built for: 12 heads of 128 over 21 x 30 x 52 tokens, 30 heads of
64 over a joint sequence, 24 heads of 128, and the 4 heads of 64 over 256
tokens of the small fp32 model.  Operands are column blocks of one projection's
output, [rows, (heads + 2 kv_heads) head_dim].

Values: queries and keys N(0, 1.2), so that a row's weights are neither flat nor
on one key, values N(0, 1), gradients N(0, 1e-2).
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
THETA = 10000.0


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _rope(rows, heads, d, axes, grid="", halves=False, first=0, dtype="bf16", far=0.0):
    """grid: the token grid, or "" for positions of the user's own, up to ``far``; first: rows that are not rotated."""
    return dict(rows=rows, heads=heads, d=d, axes=axes, grid=grid, halves=halves, first=first, dtype=dtype, far=far)


def _mha(q, k, heads, d, kv_heads=0, pad=0, frame=0, before=-1, after=-1, q_first=0, dtype="bf16"):
    """q, k: rows of each sequence; pad: rows that each sequence of keys has room for (0: packed); frame: rows of a
    frame (0: every row sees all keys of its sequence), which sees ``before`` frames before and ``after`` after it
    (-1: all); q_first: position of a sequence's first query (-1: its last query is at its last key)."""
    return dict(q=q, k=k, heads=heads, kv_heads=kv_heads or heads, d=d, pad=pad, frame=frame, before=before,
                after=after, q_first=q_first, dtype=dtype)


def listed():
    return [
        # one token's queries and keys: launch latency
        dict(name="rope 1x24x128", kind="rope", **_rope(1, 24, 128, "44,42,42", grid="1,1,1")),
        # queries and keys of a 480p clip's self-attention
        dict(name="rope 32760x24x128", kind="rope", **_rope(32760, 24, 128, "44,42,42", grid="21,30,52")),
        # the gradient of a joint sequence's queries and keys: 256 text rows, 33 frames at scaled positions
        dict(name="rope grad 67576x48x128", kind="rope_grad",
             **_rope(67576, 48, 128, "16,56,56", halves=True, first=256, far=2000.0)),
        # a single query row against the keys of a whole clip: latency
        dict(name="mha 1 of 32760", kind="mha", **_mha("1", "32760", 12, 128)),
        # the small fp32 model's self-attention
        dict(name="mha fp32 256", kind="mha", **_mha("256", "256", 4, 64, dtype="fp32")),
        # three joint sequences of different lengths in one batch
        dict(name="mha packed 4726+2501+1013", kind="mha", **_mha("4726,2501,1013", "4726,2501,1013", 30, 64)),
        # a 480p clip that is causal in its 21 latent frames
        dict(name="mha frames 32760", kind="mha", **_mha("32760", "32760", 12, 128, frame=1560, after=0)),
        # gradients of the small fp32 model
        dict(name="mha grad fp32 256", kind="mha_grad", **_mha("256", "256", 4, 64, dtype="fp32")),
        # two clips' cross-attention to text, padded to 512 rows
        dict(name="mha grad cross 32760x512", kind="mha_grad", **_mha("16380,16380", "301,512", 12, 128, pad=512)),
        # a joint sequence of 226 text and 4500 video rows
        dict(name="mha grad 4726", kind="mha_grad", **_mha("4726", "4726", 30, 64)),
        # 24 query heads on 8 key heads, a window of five frames
        dict(name="mha grad window 8190", kind="mha_grad",
             **_mha("8190", "8190", 24, 128, kv_heads=8, frame=390, before=4, after=0)),
        # the largest: self-attention of a 480p clip
        dict(name="mha grad 32760", kind="mha_grad", **_mha("32760", "32760", 12, 128)),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_rope(rng):
    d = rng.choice([64, 64, 128, 128])
    heads = rng.choice([4, 24, 48, 60])
    rows = _log(rng, 1, min(67576, 67576 * 6144 // (2 * heads * d)))
    first = rng.choice([0, 0, min(rows, rng.randint(1, 300))])
    how = dict(halves=rng.random() < 0.4, first=first, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    axes = rng.choice({64: ["24,20,20", "16,24,24", "64", "8,12,12"], 128: ["44,42,42", "16,56,56", "32,48,48", "16,24,24"]}[d])
    if rng.random() < 0.5:
        if axes.count(",") == 0:
            grid = str(max(rows - first, 1))
        else:  # a batch of clips repeats the grid, and its last one may end early
            h, w = rng.randint(1, 45), rng.randint(1, 80)
            grid = f"{rng.randint(1, 33)},{h},{w}"
        return _rope(rows, heads, d, axes, grid=grid, **how)
    return _rope(rows, heads, d, axes, far=rng.choice([50.0, 2000.0, 2e5]), **how)


def _draw_mha(rng, most):
    """``most``: products of a query and a key, over heads and head dim, that the case may have."""
    heads, kv_heads, d = rng.choice([(4, 4, 64), (12, 12, 128), (30, 30, 64), (24, 24, 128), (24, 8, 128), (12, 4, 64),
                                     (16, 1, 128)])
    dtype = "fp32" if (heads, d) == (4, 64) and rng.random() < 0.7 else "bf16"
    if dtype == "fp32":
        most = min(most, 4 * 64 * 2048 * 2048)
    count = rng.choice([1, 1, 1, 2, 3, 8])
    shape = rng.choice(["self", "self", "cross", "frames", "few"])
    pairs = most // (heads * d * count)
    pad, how = 0, {}
    if shape in ("self", "frames"):
        top = max(2, int(min(32760 // count, math.isqrt(pairs))))
        q = [_log(rng, 1, top) for _ in range(count)]
        k = list(q)
        if shape == "frames":
            frame = rng.choice([1, 16, 100, 390, 1560])
            how = dict(frame=frame, before=rng.choice([-1, 0, 2, 5]), after=rng.choice([0, 0, 1]))
    elif shape == "cross":
        k = [rng.randint(1, 512) for _ in range(count)]
        pad = rng.choice([0, 512])
        q = [_log(rng, 1, max(1, min(32760 // count, pairs // 512))) for _ in range(count)]
    else:  # a chunk of new rows against all the keys up to it
        k = [_log(rng, 64, max(65, min(32760 // count, math.isqrt(pairs)))) for _ in range(count)]
        q = [max(1, min(n, rng.choice([1, 3, 100, n // 8]))) for n in k]
        if rng.random() < 0.5:
            how = dict(frame=rng.choice([1, 64, 390]), after=0, q_first=-1)
    return _mha(",".join(map(str, q)), ",".join(map(str, k)), heads, d, kv_heads=kv_heads, pad=pad, dtype=dtype, **how)


def draw(rng):
    kind = rng.choice(["rope", "rope_grad", "mha", "mha", "mha_grad", "mha_grad"])
    if kind.startswith("rope"):
        return dict(kind=kind, **_draw_rope(rng))
    return dict(kind=kind, **_draw_mha(rng, 12 * 128 * 16000 ** 2))


def _ints(text):
    return [int(t) for t in text.split(",") if t]


def _bounds(case):
    """First row and row past the last of each sequence, of the queries and of the keys, and the rows in all."""
    q, k = _ints(case["q"]), _ints(case["k"])
    qb = np.stack([np.cumsum([0] + q[:-1]), np.cumsum(q)], 1)
    if case["pad"]:
        kb = np.array([[i * case["pad"], i * case["pad"] + n] for i, n in enumerate(k)])
        return qb, kb, sum(q), len(k) * case["pad"]
    kb = np.stack([np.cumsum([0] + k[:-1]), np.cumsum(k)], 1)
    return qb, kb, sum(q), sum(k)


def _visible(case, nq, nk):
    """First visible key and the one past the last, of each query row of a sequence."""
    i = np.arange(nq)
    if not case["frame"]:
        return np.zeros(nq, np.int64), np.full(nq, nk)
    at = (i + (case["q_first"] if case["q_first"] >= 0 else nk - nq)) // case["frame"]
    lo = np.zeros(nq, np.int64) if case["before"] < 0 else (at - case["before"]) * case["frame"]
    hi = np.full(nq, nk) if case["after"] < 0 else (at + case["after"] + 1) * case["frame"]
    return np.clip(lo, 0, nk), np.clip(hi, 0, nk)


def _pairs(case):
    """Visible products of a query and a key, over all sequences."""
    n = 0
    for q, k in zip(_ints(case["q"]), _ints(case["k"])):
        lo, hi = _visible(case, q, k)
        n += int(np.maximum(hi - lo, 0).sum())
    return n


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.empty(*shape, device=DEV, dtype=torch.float32).normal_(0, std, generator=gen).to(dtype)

    s = dict(case=case)
    if case["kind"] in ("rope", "rope_grad"):
        width = case["heads"] * case["d"]
        # queries and keys are the first two thirds of a projection's output
        s["x"] = normal(case["rows"], width + width // 2, std=1.2 if case["kind"] == "rope" else 1e-2)[:, :width]
        s["positions"] = None
        if not case["grid"]:
            axes = len(_ints(case["axes"]))
            s["positions"] = case["far"] * torch.rand(case["rows"], axes, device=DEV, generator=gen)
        return s
    h, kv, d = case["heads"], case["kv_heads"], case["d"]
    qb, kb, nq, nk = _bounds(case)
    if case["q"] == case["k"] and not case["pad"]:
        qkv = normal(nq, (h + 2 * kv) * d)
        qkv[:, :(h + kv) * d] *= 1.2
        s["q"], s["k"], s["v"] = qkv[:, :h * d], qkv[:, h * d:(h + kv) * d], qkv[:, (h + kv) * d:]
    else:
        s["q"] = normal(nq, h * d, std=1.2)
        both = normal(nk, 2 * kv * d)
        both[:, :kv * d] *= 1.2
        s["k"], s["v"] = both[:, :kv * d], both[:, kv * d:]
    s["q_bounds"] = s["k_bounds"] = None
    if len(qb) > 1 or case["pad"]:
        s["q_bounds"] = torch.from_numpy(qb.astype(np.int32)).to(DEV)
        s["k_bounds"] = torch.from_numpy(kb.astype(np.int32)).to(DEV)
    if case["kind"] == "mha_grad":
        s["dout"] = normal(nq, h * d, std=1e-2)
        forward = _plain_mha(s)
        s["out"], s["lse"] = forward["out"], forward["lse"]
        # rows that belong to no sequence keep what the user's buffers hold
        for name in ("q", "k", "v"):
            s["d" + name] = torch.zeros(s[name].shape, dtype=dtype, device=DEV)
    if own:
        from paper_2607_12358_gb300 import acid

        s["workspace"] = acid.mha_workspace(s["q"], s["k"], h, backward=case["kind"] == "mha_grad",
                                            q_bounds=s["q_bounds"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2607_12358_gb300 import acid

    c = s["case"]
    if c["kind"] in ("rope", "rope_grad"):
        call = acid.acid_rope_forward if c["kind"] == "rope" else acid.acid_rope_backward
        return call(s["x"], c["heads"], tuple(_ints(c["axes"])), theta=THETA, grid=tuple(_ints(c["grid"])) or None,
                    positions=s["positions"], first_rows=c["first"], halves=c["halves"])
    how = dict(q_bounds=s["q_bounds"], k_bounds=s["k_bounds"], frame_rows=c["frame"], frames_before=c["before"],
               frames_after=c["after"], q_first=c["q_first"], workspace=s.get("workspace"))
    if c["kind"] == "mha":
        out, lse = acid.acid_mha_forward(s["q"], s["k"], s["v"], c["heads"], **how)
        return dict(out=out, lse=lse)
    dq, dk, dv = acid.acid_mha_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], c["heads"], dq=s["dq"],
                                        dk=s["dk"], dv=s["dv"], **how)
    return dict(dq=dq, dk=dk, dv=dv)


def _run_plain(s):
    return {"rope": _plain_rope, "rope_grad": _plain_rope, "mha": _plain_mha, "mha_grad": _plain_mha_grad}[
        s["case"]["kind"]](s)


def _positions(s):
    """Positions of the rotated rows along each axis, in 64 bits."""
    c = s["case"]
    if s["positions"] is not None:
        return s["positions"][c["first"]:].double()
    n, out = torch.arange(c["rows"] - c["first"], device=DEV), []
    for size in reversed(_ints(c["grid"])):
        out.append(n % size)
        n = n // size
    return torch.stack(out[::-1], 1).double()


def _plain_rope(s):
    c = s["case"]
    dims, first = _ints(c["axes"]), c["first"]
    at = _positions(s)
    angle = torch.cat([at[:, a:a + 1] * THETA ** (-torch.arange(0, n, 2, device=DEV, dtype=torch.float64) / n)
                       for a, n in enumerate(dims)], 1)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["kind"] == "rope_grad":
        sin = -sin
    x = s["x"].float().reshape(c["rows"], c["heads"], c["d"])
    out, turned = x.clone(), sum(dims)
    if c["halves"]:
        a, b = x[first:, :, :turned // 2], x[first:, :, turned // 2:turned]
        out[first:, :, :turned // 2] = a * cos - b * sin
        out[first:, :, turned // 2:turned] = a * sin + b * cos
    else:
        a, b = x[first:, :, 0:turned:2], x[first:, :, 1:turned:2]
        out[first:, :, 0:turned:2] = a * cos - b * sin
        out[first:, :, 1:turned:2] = a * sin + b * cos
    return out.to(DTYPES[c["dtype"]]).reshape(c["rows"], -1)


def _heads(t, a, e, heads, d):
    """Rows a .. e - 1 as [heads, rows, d] in fp32."""
    return t[a:e].float().view(e - a, heads, d).transpose(0, 1)


def _chunks(nq, nk, heads):
    """Query rows taken at a time: up to 1 GB of scores."""
    step = max(1, (1 << 28) // max(1, heads * nk))
    return [(a, min(nq, a + step)) for a in range(0, nq, step)]


def _hidden(c, nq, nk, a, e):
    """[e - a, nk] truth values: key not visible; None if all are."""
    if not c["frame"]:
        return None
    lo, hi = (torch.from_numpy(t[a:e]).to(DEV)[:, None] for t in _visible(c, nq, nk))
    j = torch.arange(nk, device=DEV)
    return (j < lo) | (j >= hi)


def _plain_mha(s):
    c = s["case"]
    h, kv, d = c["heads"], c["kv_heads"], c["d"]
    qb, kb, rows, _ = _bounds(c)
    out = torch.zeros(rows, h * d, dtype=DTYPES[c["dtype"]], device=DEV)
    lse = torch.zeros(h, rows, device=DEV)
    for (qa, qe), (ka, ke) in zip(qb.tolist(), kb.tolist()):
        k, v = _heads(s["k"], ka, ke, kv, d)[:, None], _heads(s["v"], ka, ke, kv, d)[:, None]
        for a, e in _chunks(qe - qa, ke - ka, h):
            q = _heads(s["q"], qa + a, qa + e, h, d).reshape(kv, h // kv, e - a, d)
            p = (q @ k.transpose(2, 3)).mul_(d ** -0.5)
            hidden = _hidden(c, qe - qa, ke - ka, a, e)
            if hidden is not None:
                p.masked_fill_(hidden, -math.inf)
            top = p.amax(3, keepdim=True)
            top = torch.where(top == -math.inf, 0, top)
            p = p.sub_(top).exp_()
            total = p.sum(3, keepdim=True)
            o = (p @ v) / torch.where(total == 0, 1, total)
            out[qa + a:qa + e] = o.view(h, e - a, d).transpose(0, 1).reshape(e - a, -1).to(out.dtype)
            lse[:, qa + a:qa + e] = (top + total.log()).view(h, e - a)
    return dict(out=out, lse=lse)


def _plain_mha_grad(s):
    c = s["case"]
    h, kv, d = c["heads"], c["kv_heads"], c["d"]
    scale = d ** -0.5
    qb, kb, nq, nk = _bounds(c)
    dtype = DTYPES[c["dtype"]]
    dq = torch.zeros(nq, h * d, dtype=dtype, device=DEV)
    dk, dv = (torch.zeros(nk, kv * d, dtype=dtype, device=DEV) for _ in range(2))
    for (qa, qe), (ka, ke) in zip(qb.tolist(), kb.tolist()):
        k, v = _heads(s["k"], ka, ke, kv, d)[:, None], _heads(s["v"], ka, ke, kv, d)[:, None]
        sum_k, sum_v = torch.zeros(kv, ke - ka, d, device=DEV), torch.zeros(kv, ke - ka, d, device=DEV)
        for a, e in _chunks(qe - qa, ke - ka, h):
            q, g, o = (_heads(s[n], qa + a, qa + e, h, d).reshape(kv, h // kv, e - a, d) for n in ("q", "dout", "out"))
            lse = s["lse"][:, qa + a:qa + e].reshape(kv, h // kv, e - a, 1)
            p = (q @ k.transpose(2, 3)).mul_(scale)
            hidden = _hidden(c, qe - qa, ke - ka, a, e)
            if hidden is not None:
                p.masked_fill_(hidden, -math.inf)
            p = p.sub_(torch.where(lse == -math.inf, 0, lse)).exp_()
            sum_v += (p.transpose(2, 3) @ g).sum(1)
            dp = g @ v.transpose(2, 3)
            ds = dp.sub_((g * o).sum(3, keepdim=True)).mul_(p)
            part = (ds @ k).mul_(scale).view(h, e - a, d)
            dq[qa + a:qa + e] = part.transpose(0, 1).reshape(e - a, -1).to(dtype)
            sum_k += (ds.transpose(2, 3) @ q).sum(1)
        dk[ka:ke] = (sum_k * scale).transpose(0, 1).reshape(ke - ka, -1).to(dtype)
        dv[ka:ke] = sum_v.transpose(0, 1).reshape(ke - ka, -1).to(dtype)
    return dict(dq=dq, dk=dk, dv=dv)


# ---------------------------------------------------------------------------
# the work of one pass
# ---------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] in ("rope", "rope_grad"):
        n = case["rows"] * case["heads"] * case["d"]
        table = 0 if case["grid"] else 4 * case["rows"] * len(_ints(case["axes"]))
        return {"bytes": 2 * size * n + table, "flops": 3 * n}
    h, kv, d = case["heads"], case["kv_heads"], case["d"]
    nq, nk = sum(_ints(case["q"])), sum(_ints(case["k"]))
    products = _pairs(case) * h * d
    if case["kind"] == "mha":
        return {"bytes": size * d * (2 * h * nq + 2 * kv * nk) + 4 * h * nq, "flops": 4 * products}
    return {"bytes": size * d * (4 * h * nq + 4 * kv * nk) + 4 * h * nq, "flops": 10 * products}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] in ("rope", "rope_grad"):
        return _exact_rope(prepare(case, seed))
    if work(case)["flops"] > 6e12:  # products in 64 bits run at about 1e12 a second
        return None
    s = prepare(case, seed)
    return _exact_mha(s) if case["kind"] == "mha" else _exact_mha_grad(s)


def _exact_rope(s):
    """Each pair as a complex number times e^(i angle)."""
    c = s["case"]
    x = s["x"].double().reshape(c["rows"], c["heads"], c["d"])
    out = x.clone()
    dims = _ints(c["axes"])
    at, turned, pair = _positions(s), sum(dims), 0
    for a, n in enumerate(dims):
        for j in range(n // 2):
            i, k = (pair, pair + turned // 2) if c["halves"] else (2 * pair, 2 * pair + 1)
            angle = at[:, a] * THETA ** (-2 * j / n)
            turn = torch.polar(torch.ones_like(angle), -angle if c["kind"] == "rope_grad" else angle)
            z = torch.complex(x[c["first"]:, :, i], x[c["first"]:, :, k]) * turn[:, None]
            out[c["first"]:, :, i], out[c["first"]:, :, k] = z.real, z.imag
            pair += 1
    return out.reshape(c["rows"], -1)


def _each_head(s):
    """(head, shared head, rows of queries, rows of keys, scores' hidden places) of every sequence, some rows at a time."""
    c = s["case"]
    qb, kb, _, _ = _bounds(c)
    for (qa, qe), (ka, ke) in zip(qb.tolist(), kb.tolist()):
        for a, e in _chunks(qe - qa, ke - ka, 4):
            hidden = _hidden(c, qe - qa, ke - ka, a, e)
            for head in range(c["heads"]):
                yield head, head * c["kv_heads"] // c["heads"], slice(qa + a, qa + e), slice(ka, ke), hidden


def _exact_weights(s, head, shared, rows, keys, hidden):
    d = s["case"]["d"]
    q = s["q"][rows, head * d:(head + 1) * d].double()
    k = s["k"][keys, shared * d:(shared + 1) * d].double()
    score = q @ k.T / math.sqrt(d)
    if hidden is not None:
        score = score.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(score, 1)
    return torch.exp(score - torch.where(lse == -math.inf, 0, lse)[:, None]), lse, q, k


def _exact_mha(s):
    c = s["case"]
    d, rows = c["d"], s["q"].shape[0]
    out = torch.zeros(rows, c["heads"] * d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["heads"], rows, dtype=torch.float64, device=DEV)
    for head, shared, at, keys, hidden in _each_head(s):
        p, total, _, _ = _exact_weights(s, head, shared, at, keys, hidden)
        out[at, head * d:(head + 1) * d] = p @ s["v"][keys, shared * d:(shared + 1) * d].double()
        lse[head, at] = total
    return dict(out=out, lse=lse)


def _exact_mha_grad(s):
    """With p the weights: dv = p^T g, and the score's gradient is p (g v^T) less p times the row's sum of it."""
    c = s["case"]
    d = c["d"]
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in ("q", "k", "v"))
    for head, shared, at, keys, hidden in _each_head(s):
        p, _, q, k = _exact_weights(s, head, shared, at, keys, hidden)
        mine, its = slice(head * d, (head + 1) * d), slice(shared * d, (shared + 1) * d)
        g = s["dout"][at, mine].double()
        dv[keys, its] += p.T @ g
        along = p * (g @ s["v"][keys, its].double().T)
        ds = (along - p * along.sum(1, keepdim=True)) / math.sqrt(d)
        dq[at, mine] = ds @ k
        dk[keys, its] += ds.T @ q
    return dict(dq=dq, dk=dk, dv=dv)
