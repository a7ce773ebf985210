"""The adaLN operators whose speed this repository answers for, as a user's program calls them.

Two operators around a DiT branch, and what belongs to them:

* the norm site between two branches: the branch's output is normed (sandwich
  norm), gated and added to the scaled residual stream, and the sum is normed
  and modulated for the next branch, in one pass; with the gradients of every
  input, as a fine-tuning or calibration step needs them;
* the modulation projection of the site's shift, scale and gate vectors,
  W SiLU(temb) + b, from a weight held in 4 bits with a scale (and optionally a
  zero point) for each group of columns: the product for one or a few timestep
  embeddings, the gradient of its input (the 4-bit weight itself is frozen) and
  of its bias, and the quantiser that lays the weight out.

Widths and token counts are the ones of the shapes this repository is built for
(256, 1536, 1920 and 3072 columns; 480p and 720p token grids), text rows first.
A group of rows with modulation vectors of its own is the text, the video, or
one latent frame where every frame has its own timestep.

Values: hidden states N(0.2, 1) with a few channels 20 times as large, branch
outputs N(0, 0.5), modulation vectors N(0, 0.3), gradients N(0, 1e-2),
weights N(0, 0.02).
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _site(rows, d, stream, branch, post, pre, first=0, group=0, tanh=False, weights=True):
    return dict(rows=rows, d=d, stream=stream, branch=branch, post=post, pre=pre, first=first, group=group, tanh=tanh,
                weights=weights)


def _weight(n, k, group, zeros, scales):
    return dict(n=n, k=k, group=group, zeros=zeros, scales=scales)


def listed():
    return [
        # one token through a site of a 1536-wide model: launch latency
        dict(name="site 1x1536", kind="site", **_site(1, 1536, "fp32", "fp32", "rms", "layer")),
        # a 480p clip's site: fp32 stream as inside the blocks, one timestep for all rows
        dict(name="site 32760x1536", kind="site", **_site(32760, 1536, "fp32", "bf16", "rms", "layer")),
        # the largest: 256 text rows and 33 latent frames with a timestep each, bf16 stream
        dict(name="site frames 67576x3072", kind="site",
             **_site(67576, 3072, "bf16", "bf16", "rms", "rms", first=256, group=2040, tanh=True)),
        # gradients at the 226 text rows of a joint sequence
        dict(name="site grad 226x1920", kind="site_grad", **_site(226, 1920, "bf16", "bf16", "layer", "layer")),
        # gradients at a 480p clip's site, 21 latent frames with a timestep each
        dict(name="site grad 32760x1536", kind="site_grad",
             **_site(32760, 1536, "fp32", "bf16", "rms", "layer", group=1560)),
        # one block's six modulation vectors from one timestep embedding
        dict(name="q4 9216x1536 m1", kind="q4", m=1, x="fp32", out="fp32", silu=True,
             **_weight(9216, 1536, 128, False, "bf16")),
        # the vectors of all 30 blocks of a step in one call
        dict(name="q4 276480x1536 m1", kind="q4", m=1, x="fp32", out="fp32", silu=True,
             **_weight(276480, 1536, 64, True, "bf16")),
        # twelve vectors of a 3072-wide joint block for the text and 33 frames
        dict(name="q4 36864x3072 m34", kind="q4", m=34, x="fp32", out="fp32", silu=True,
             **_weight(36864, 3072, 128, False, "bf16")),
        # the timestep embedding's gradient through one block's projection
        dict(name="q4 grad 9216x1536 m1", kind="q4_grad", m=1, x="fp32", silu=True,
             **_weight(9216, 1536, 128, False, "bf16")),
        # the same for the text and 33 frames of a 3072-wide block
        dict(name="q4 grad 18432x3072 m34", kind="q4_grad", m=34, x="fp32", silu=True,
             **_weight(18432, 3072, 64, True, "fp32")),
        # a final layer's two vectors quantised, and its values read back for the error
        dict(name="quantise 3072x1536", kind="quantise", **_weight(3072, 1536, 32, True, "bf16")),
        # a 3072-wide block's twelve vectors
        dict(name="quantise 36864x3072", kind="quantise", **_weight(36864, 3072, 128, False, "bf16")),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["site", "site", "site_grad", "site_grad", "q4", "q4", "q4_grad", "quantise"])
    if kind in ("site", "site_grad"):
        d = rng.choice([256, 1000, 1536, 1920, 3072])
        rows = _log(rng, 1, int(67576 * 3072 / d * (0.25 if kind == "site_grad" else 0.5)))
        first = rng.choice([0, 0, min(rows, rng.randint(1, 512))])
        # one group, one a frame, or (a few rows) one a row
        group = rng.choice([0, 0, max(16, rows // rng.randint(2, 33)), 1 if rows <= 2048 else 0])
        stream, branch = rng.choice([("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"),
                                     ("bf16", "fp32")])
        return dict(kind=kind, **_site(rows, d, stream, branch, rng.choice(["none", "rms", "rms", "layer"]),
                                       rng.choice(["rms", "layer", "layer"]), first=first, group=group,
                                       tanh=rng.random() < 0.3, weights=rng.random() < 0.7))
    k = rng.choice([256, 1000, 1536, 1920, 3072])
    n = _log(rng, 64, min(276480, 36864 * 3072 // k))
    w = _weight(n, k, rng.choice([32, 64, 128, 128]), rng.random() < 0.4, rng.choice(["bf16", "fp32"]))
    if kind == "quantise":  # with a scale of 32 bits a quotient in the middle of two codes depends on its last bit
        return dict(kind=kind, **dict(w, scales="bf16"))
    m = _log(rng, 1, 64)
    if kind == "q4":
        return dict(kind=kind, m=m, x=rng.choice(["fp32", "fp32", "bf16"]), out=rng.choice(["fp32", "fp32", "bf16"]),
                    silu=rng.random() < 0.8, **w)
    return dict(kind=kind, m=m, x=rng.choice(["fp32", "fp32", "bf16"]), silu=rng.random() < 0.8, **w)


def _groups(case):
    rest = case["rows"] - case["first"]
    group = case["group"] or max(rest, 1)
    return (1 if case["first"] else 0) + -(-rest // group)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.empty(*shape, device=DEV, dtype=torch.float32).normal_(mean, std, generator=gen).to(dtype)

    if case["kind"] in ("site", "site_grad"):
        rows, d, groups = case["rows"], case["d"], _groups(case)
        stream, branch = DTYPES[case["stream"]], DTYPES[case["branch"]]
        s = dict(case=case)
        x = normal(rows, d, mean=0.2)
        x[:, torch.randint(0, d, (4,), device=DEV, generator=gen)] *= 20
        # the vectors come as one projection's output, [groups, 3 d]
        mod = normal(groups, 3 * d, std=0.3)
        s["shift"], s["scale"], s["gate"] = mod[:, :d], mod[:, d:2 * d], mod[:, 2 * d:]
        s["post_w"] = normal(d, mean=1.0, std=0.1) if case["weights"] else None
        s["pre_w"] = normal(d, mean=1.0, std=0.1) if case["weights"] else None
        s["y"] = normal(rows, d, std=0.5, dtype=branch)
        if case["kind"] == "site":
            s["x"] = x.to(stream)
        else:
            s["r"] = x.to(stream)
            s["du"] = normal(rows, d, std=1e-2, dtype=branch)
            s["dr"] = normal(rows, d, std=1e-2, dtype=stream)
        return s
    n, k, group = case["n"], case["k"], case["group"]
    if case["kind"] == "quantise":
        return dict(case=case, w=normal(n, k, std=0.02, dtype=torch.bfloat16))
    per_row = -(-k // group)
    s = dict(case=case)
    # 128 columns are 64 bytes: 16 words, of which word 4 t + i holds columns 32 i + 8 t .. + 7, lowest bits first;
    # what is past the last column is never used
    s["packed"] = torch.randint(-128, 128, (n, 64 * -(-k // 128)), device=DEV, generator=gen,
                                dtype=torch.int8).view(torch.uint8)
    s["scales"] = (0.006 * torch.rand(n, per_row, device=DEV, generator=gen) + 0.003).to(DTYPES[case["scales"]])
    s["zeros"] = torch.randint(5, 11, (n, per_row), device=DEV, generator=gen,
                               dtype=torch.int8).view(torch.uint8) if case["zeros"] else None
    s["x"] = normal(case["m"], k, dtype=DTYPES[case["x"]])
    if case["kind"] == "q4":
        s["bias"] = normal(n, std=0.02)
    else:
        s["g"] = normal(case["m"], n, std=1e-2)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2607_12358_gb300 import acid

    c = s["case"]
    if c["kind"] in ("site", "site_grad"):
        how = dict(gate=s["gate"], scale=s["scale"], shift=s["shift"], post_w=s["post_w"], pre_w=s["pre_w"],
                   post_norm=c["post"], pre_norm=c["pre"], eps=EPS, res_scale=0.9, branch_scale=1.1,
                   gate_tanh=c["tanh"], first_rows=c["first"], group_rows=c["group"])
        if c["kind"] == "site":
            r, u = acid.acid_norm_site_forward(s["x"], s["y"], **how)
            return dict(r=r, u=u)
        g = acid.acid_norm_site_backward(s["du"], s["r"], s["y"], dr=s["dr"], **how)
        return {name: g[name] for name in ("dx", "dy", "dgate", "dscale", "dshift", "dpost_w", "dpre_w")
                if name in g and g[name] is not None}
    if c["kind"] == "quantise":
        q = acid.acid_q4_quantize(s["w"], c["group"], zeros=c["zeros"], scale_dtype=DTYPES[c["scales"]])
        return dict(values=acid.acid_q4_dequantize(q, torch.float32), scales=q.scales)
    q = acid.Q4Weight(s["packed"], s["scales"], s["zeros"], c["n"], c["k"], c["group"])
    if c["kind"] == "q4":
        return acid.acid_q4_linear_forward(s["x"], q, s["bias"], silu=c["silu"], out_dtype=DTYPES[c["out"]])
    dx, dbias = acid.acid_q4_linear_backward(s["g"], q, s["x"], silu=c["silu"])
    return dict(dx=dx, dbias=dbias)


def _run_plain(s):
    return {"site": _plain_site, "site_grad": _plain_site_grad, "quantise": _plain_quantise, "q4": _plain_q4,
            "q4_grad": _plain_q4_grad}[s["case"]["kind"]](s)


def _row_groups(c):
    i = torch.arange(c["rows"], device=DEV)
    group = c["group"] or max(c["rows"] - c["first"], 1)
    return torch.where(i < c["first"], 0, (1 if c["first"] else 0) + (i - c["first"]) // group)


def _normed(v, kind):
    """v normed along its rows, and 1 over the root that it was divided by."""
    if kind == "none":
        return v, None
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    inv = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * inv, inv


def _plain_site(s):
    c = s["case"]
    at = _row_groups(c)
    gate = torch.tanh(s["gate"]) if c["tanh"] else s["gate"]
    z, _ = _normed(s["y"].float(), c["post"])
    if s["post_w"] is not None:
        z = z * s["post_w"]
    r = 0.9 * s["x"].float() + 1.1 * gate[at] * z
    u, _ = _normed(r, c["pre"])
    if s["pre_w"] is not None:
        u = u * s["pre_w"]
    u = u * (1 + s["scale"][at]) + s["shift"][at]
    return dict(r=r.to(DTYPES[c["stream"]]), u=u.to(DTYPES[c["branch"]]))


def _group_sums(v, c):
    """[groups, d] sums of v over the rows of each group."""
    first, group = c["first"], c["group"] or max(c["rows"] - c["first"], 1)
    head = v[:first].sum(0, keepdim=True)[:1 if first else 0]
    rest = torch.nn.functional.pad(v[first:], (0, 0, 0, -(c["rows"] - first) % group))
    return torch.cat([head, rest.view(-1, group, v.shape[1]).sum(1)])


def _back(dn, n, inv, kind):
    """The gradient of a norm's input from dn, that of its output n."""
    if kind == "none":
        return dn
    out = dn - n * (dn * n).mean(1, keepdim=True)
    if kind == "layer":
        out = out - dn.mean(1, keepdim=True)
    return out * inv


def _plain_site_grad(s):
    c = s["case"]
    at = _row_groups(c)
    one = torch.ones(c["d"], device=DEV)
    post_w = one if s["post_w"] is None else s["post_w"]
    pre_w = one if s["pre_w"] is None else s["pre_w"]
    gate = torch.tanh(s["gate"]) if c["tanh"] else s["gate"]
    du = s["du"].float()
    n, inv = _normed(s["r"].float(), c["pre"])
    out = dict(dshift=_group_sums(du, c), dscale=_group_sums(du * n * pre_w, c))
    scaled = du * (1 + s["scale"][at])
    if s["pre_w"] is not None:
        out["dpre_w"] = (scaled * n).sum(0)
    dr = s["dr"].float() + _back(scaled * pre_w, n, inv, c["pre"])
    out["dx"] = (0.9 * dr).to(DTYPES[c["stream"]])
    p, inv = _normed(s["y"].float(), c["post"])
    out["dgate"] = _group_sums(1.1 * dr * p * post_w, c) * (1 - gate * gate if c["tanh"] else 1)
    dz = 1.1 * dr * gate[at]
    if s["post_w"] is not None:
        out["dpost_w"] = (dz * p).sum(0)
    out["dy"] = _back(dz * post_w, p, inv, c["post"]).to(DTYPES[c["branch"]])
    return out


def _values(s):
    """The 4-bit weight's values [n, k]."""
    c = s["case"]
    words = s["packed"].view(torch.int32).view(c["n"], -1, 4, 4).transpose(2, 3).unsqueeze(-1)
    codes = (words >> torch.arange(0, 32, 4, device=DEV, dtype=torch.int32)) & 15
    codes = codes.reshape(c["n"], -1)[:, :c["k"]]
    zeros = 8 if s["zeros"] is None else s["zeros"].int().repeat_interleave(c["group"], 1)[:, :c["k"]]
    return (codes - zeros) * s["scales"].float().repeat_interleave(c["group"], 1)[:, :c["k"]]


def _plain_q4(s):
    c = s["case"]
    x = s["x"].float()
    if c["silu"]:
        x = x / (1 + torch.exp(-x))
    return (x @ _values(s).T + s["bias"]).to(DTYPES[c["out"]])


def _plain_q4_grad(s):
    c = s["case"]
    x = s["x"].float()
    dx = s["g"] @ _values(s)
    if c["silu"]:
        e = 1 / (1 + torch.exp(-x))
        dx = dx * (e * (1 + x * (1 - e)))
    return dict(dx=dx.to(DTYPES[c["x"]]), dbias=s["g"].sum(0))


def _plain_quantise(s):
    c = s["case"]
    n, k, group = c["n"], c["k"], c["group"]
    per_row = -(-k // group)
    w = torch.nn.functional.pad(s["w"].float(), (0, per_row * group - k)).view(n, per_row, group)
    if c["zeros"]:
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        scales = ((hi - lo) / 15).to(DTYPES[c["scales"]])
        step = torch.where(scales == 0, 1, scales.float())
        zero = torch.round(-lo / step).clamp(0, 15)
        codes = (torch.round(w / step[:, :, None]) + zero[:, :, None]).clamp(0, 15)
    else:
        scales = (w.abs().amax(2) / 7).to(DTYPES[c["scales"]])
        step = torch.where(scales == 0, 1, scales.float())
        zero = torch.full_like(step, 8)
        codes = torch.round(w / step[:, :, None]).clamp(-8, 7) + 8
    values = (codes - zero[:, :, None]) * scales.float()[:, :, None]
    return dict(values=values.reshape(n, -1)[:, :k].contiguous(), scales=scales)


# ---------------------------------------------------------------------------
# the work of one pass
# ---------------------------------------------------------------------------

def work(case):
    if case["kind"] in ("site", "site_grad"):
        stream, branch = (4 if case[t] == "fp32" else 2 for t in ("stream", "branch"))
        elems, vectors = case["rows"] * case["d"], 4 * case["d"]
        if case["kind"] == "site":  # x, y, shift, scale, gate and the weights read, r and u written
            return dict(bytes=elems * 2 * (stream + branch) + vectors * (3 * _groups(case) + 2 * case["weights"]),
                        flops=20 * elems)
        # r, dr, y, du, scale and gate read; dx, dy and the vectors' gradients written
        return dict(bytes=elems * 3 * (stream + branch) + vectors * (5 * _groups(case) + 4 * case["weights"]),
                    flops=40 * elems)
    n, k = case["n"], case["k"]
    per_row = -(-k // case["group"])
    weight = n * k / 2 + n * per_row * ((4 if case["scales"] == "fp32" else 2) + (1 if case["zeros"] else 0))
    if case["kind"] == "quantise":  # bf16 weight read, 4 bits and scales written, fp32 values written
        return dict(bytes=6 * n * k + weight, flops=6 * n * k)
    m, x = case["m"], 4 if case["x"] == "fp32" else 2
    if case["kind"] == "q4":
        return dict(bytes=weight + m * k * x + 4 * n + m * n * (4 if case["out"] == "fp32" else 2), flops=2 * m * n * k)
    return dict(bytes=weight + 2 * m * k * x + 4 * m * n + 4 * n, flops=2 * m * n * k)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"site": _exact_site, "site_grad": _exact_site_grad, "q4": _exact_q4, "q4_grad": _exact_q4_grad,
            "quantise": _exact_quantise}[case["kind"]](s, case)


def _segments(case):
    """(first row, end row) of each group."""
    cuts, at = [], 0
    if case["first"]:
        cuts.append((0, case["first"]))
        at = case["first"]
    while at < case["rows"]:
        end = min(case["rows"], at + (case["group"] or case["rows"]))
        cuts.append((at, end))
        at = end
    return cuts


def _unit(v, kind):
    """(v normed, standard deviation with epsilon) in the definition's own terms."""
    if kind == "none":
        return v, torch.ones_like(v[:, :1])
    centred = v - v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else v
    dev = torch.sqrt(centred.pow(2).sum(1, keepdim=True) / v.shape[1] + EPS)
    return centred / dev, dev


def _exact_site(s, case):
    r, u = (torch.empty(case["rows"], case["d"], dtype=torch.float64, device=DEV) for _ in range(2))
    for b, (a, e) in enumerate(_segments(case)):
        gate = s["gate"][b].double()
        gate = gate.tanh() if case["tanh"] else gate
        z = _unit(s["y"][a:e].double(), case["post"])[0]
        z = z * s["post_w"].double() if s["post_w"] is not None else z
        r[a:e] = s["x"][a:e].double() * 0.9 + z * gate * 1.1
        v = _unit(r[a:e], case["pre"])[0]
        v = v * s["pre_w"].double() if s["pre_w"] is not None else v
        u[a:e] = v * (s["scale"][b].double() + 1) + s["shift"][b].double()
    return dict(r=r, u=u)


def _exact_site_grad(s, case):
    rows, d, groups = case["rows"], case["d"], _groups(case)
    f64 = dict(dtype=torch.float64, device=DEV)
    out = dict(dx=torch.empty(rows, d, **f64), dy=torch.empty(rows, d, **f64))
    for name in ("dgate", "dscale", "dshift"):
        out[name] = torch.empty(groups, d, **f64)
    w = {name: torch.ones(d, **f64) if s[name] is None else s[name].double() for name in ("post_w", "pre_w")}
    dw = {name: torch.zeros(d, **f64) for name in w}

    def through(v, kind, grad):
        """grad of a norm's output taken back to its input: (grad - mean - unit mean(grad unit)) / dev."""
        unit, dev = _unit(v, kind)
        if kind == "none":
            return unit, grad
        along = (grad * unit).sum(1, keepdim=True) / d
        mean = grad.sum(1, keepdim=True) / d if kind == "layer" else 0
        return unit, (grad - mean - unit * along) / dev

    for b, (a, e) in enumerate(_segments(case)):
        raw = s["gate"][b].double()
        gate, slope = (raw.tanh(), 1 / raw.cosh() ** 2) if case["tanh"] else (raw, 1)
        scale, du = 1 + s["scale"][b].double(), s["du"][a:e].double()
        unit, back = through(s["r"][a:e].double(), case["pre"], du * (scale * w["pre_w"]))
        out["dshift"][b] = du.sum(0)
        along = (du * unit).sum(0)
        out["dscale"][b] = along * w["pre_w"]
        dw["pre_w"] += along * scale
        dr = s["dr"][a:e].double() + back
        out["dx"][a:e] = dr * 0.9
        unit, out["dy"][a:e] = through(s["y"][a:e].double(), case["post"], dr * (1.1 * gate * w["post_w"]))
        along = (dr * unit).sum(0) * 1.1
        out["dgate"][b] = along * w["post_w"] * slope
        dw["post_w"] += along * gate
    for name in w:
        if s[name] is not None:
            out["d" + name] = dw[name]
    return out


def _exact_columns(s, case, a, e):
    """Columns a .. e - 1 (within one group of the scales) of the weight in 64 bits."""
    b = s["packed"].long()
    cols = torch.arange(a, e, device=DEV)
    word = 16 * (cols // 128) + 4 * (cols % 32 // 8) + cols % 128 // 32
    byte = 4 * word + cols % 8 // 2
    codes = torch.where(cols % 2 == 0, b[:, byte] % 16, b[:, byte] // 16)
    zero = 8 if s["zeros"] is None else s["zeros"][:, a // case["group"], None].long()
    return (codes - zero).double() * s["scales"][:, a // case["group"], None].double()


def _spans(case):
    return [(a, min(case["k"], a + case["group"])) for a in range(0, case["k"], case["group"])]


def _exact_q4(s, case):
    x = s["x"].double()
    x = x * torch.sigmoid(x) if case["silu"] else x
    out = s["bias"].double().repeat(case["m"], 1)
    for a, e in _spans(case):
        out += x[:, a:e] @ _exact_columns(s, case, a, e).T
    return out


def _exact_q4_grad(s, case):
    g, x = s["g"].double(), s["x"].double()
    dx = torch.cat([g @ _exact_columns(s, case, a, e) for a, e in _spans(case)], 1)
    if case["silu"]:
        y = torch.sigmoid(x)
        dx = dx * (y + x * y * (1 - y))
    return dict(dx=dx, dbias=g.sum(0))


def _exact_quantise(s, case):
    w = s["w"].double()
    values, scales = torch.empty_like(w), []
    for a, e in _spans(case):
        v = w[:, a:e]
        lo, hi = v.min(1).values.clamp(max=0), v.max(1).values.clamp(min=0)
        span = (hi - lo) / 15 if case["zeros"] else torch.maximum(hi, -lo) / 7
        step = span.to(DTYPES[case["scales"]]).double()  # the scale is the one that is stored
        scales.append(step)
        safe = torch.where(step > 0, step, 1)
        zero = torch.round(-lo / safe).clamp(0, 15) if case["zeros"] else torch.full_like(step, 8)
        codes = (torch.round(v / safe[:, None]) + zero[:, None]).clamp(0, 15)
        values[:, a:e] = (codes - zero[:, None]) * step[:, None]
    return dict(values=values, scales=torch.stack(scales, 1))
