"""A sandwich-normed adaLN block whose modulation is held in 4 bits, and its calibration.

The block runs the norm sites and the 4-bit projections as they are meant to be used together.  With one timestep
embedding a latent frame (temb [frames, d]; the rows of a frame share their modulation):

    shift1, scale1, gate1, shift2, scale2, gate2 = W_mod SiLU(temb) + b_mod       one 4-bit projection, [frames, 6 d]
    u1     = LN(x) (1 + scale1) + shift1                                          site before the attention
    y1     = W_out attention(W_qkv u1)
    r1, u2 = x + gate1 (RMS(y1) w1), LN(r1) (1 + scale2) + shift2                 site between the branches
    y2     = W_fc2 GELU(W_fc1 u2)
    r2     = r1 + gate2 (RMS(y2) w2)                                              site after them

W_mod has 6 d^2 of the block's weights: in 4 bits it is read in a quarter of the time.  What its rounding does to the
sites' outputs is taken back, as far as a bias can, by ``calibrate``: the full-precision block's branch outputs are
recorded once, the sites are run with the 4-bit vectors, and the gradient of the squared error of their outputs goes
through the sites (acid_norm_site_backward) and through the projection (acid_q4_linear_backward) to b_mod and to temb.

    python -m paper_2607_12358_gb300.adaln --d 1536 --heads 12 --frames 21 --tokens 390 --group 64 --zeros

prints the block's error before and after the calibration as one JSON line.
"""

from __future__ import annotations

import argparse
import json

import torch

from . import acid


def random_weights(d: int, hidden: int, seed: int = 0, device="cuda") -> dict:
    """Weights of one block: fp32 modulation, bf16 branches, fp32 biases and norm weights."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (std * torch.randn(*shape, device=device, dtype=torch.float32, generator=gen)).to(dtype)

    w = dict(mod_w=normal(6 * d, d, std=0.02), mod_b=normal(6 * d, std=0.1), w1=1 + normal(d, std=0.1),
             w2=1 + normal(d, std=0.1))
    for name, n, k in (("qkv", 3 * d, d), ("out", d, d), ("fc1", hidden, d), ("fc2", d, hidden)):
        w[name] = normal(n, k, std=k ** -0.5, dtype=torch.bfloat16)
        w[name + "_b"] = normal(n, std=0.02)
    return w


class AdaLNBlock:
    """The block above.  ``group`` and ``zeros``: how the modulation's weight is quantised (acid_q4_quantize); ``group``
    None keeps it in full precision.  The bias ``mod_b`` is the block's own copy, so that it can be calibrated; so is the
    attention's workspace: a block runs on one stream at a time."""

    def __init__(self, weights: dict, heads: int, group: int | None = 64, zeros: bool = True):
        self.w, self.heads, self.d = weights, heads, weights["out"].shape[0]
        self.mod_b = weights["mod_b"].clone()
        self.mod_q4 = None if group is None else acid.acid_q4_quantize(weights["mod_w"], group, zeros)
        size = acid.attention_workspace_size(self.d // heads)
        self.attn_ws = torch.empty(size, dtype=torch.uint8, device=self.mod_b.device)

    def modulation(self, temb: torch.Tensor) -> torch.Tensor:
        """[frames, 6 d] from temb [frames, d] (fp32)."""
        if self.mod_q4 is not None:
            return acid.acid_q4_linear_forward(temb, self.mod_q4, self.mod_b, silu=True)
        return acid.acid_linear_forward(torch.nn.functional.silu(temb), self.w["mod_w"], self.mod_b)

    def vectors(self, mod: torch.Tensor) -> dict:
        names = ("shift1", "scale1", "gate1", "shift2", "scale2", "gate2")
        return {n: mod[:, i * self.d:(i + 1) * self.d] for i, n in enumerate(names)}

    # the keywords of the three sites, the same in both directions
    def _first(self, v, frame_rows):
        return dict(scale=v["scale1"], shift=v["shift1"], post_norm="none", group_rows=frame_rows)

    def _middle(self, v, frame_rows):
        return dict(gate=v["gate1"], scale=v["scale2"], shift=v["shift2"], post_w=self.w["w1"], group_rows=frame_rows)

    def _last(self, v, frame_rows):
        return dict(gate=v["gate2"], post_w=self.w["w2"], pre_norm="none", group_rows=frame_rows)

    def attention(self, u: torch.Tensor) -> torch.Tensor:
        w, d = self.w, self.d
        qkv = acid.acid_linear_forward(u, w["qkv"], w["qkv_b"])
        a = acid.acid_attention_forward(qkv[:, :d], qkv[:, d:2 * d], qkv[:, 2 * d:], self.heads, workspace=self.attn_ws)
        return acid.acid_linear_forward(a, w["out"], w["out_b"])

    def mlp(self, u: torch.Tensor) -> torch.Tensor:
        h = acid.acid_linear_forward(u, self.w["fc1"], self.w["fc1_b"], "gelu")
        return acid.acid_linear_forward(h, self.w["fc2"], self.w["fc2_b"])

    def sites(self, x, y1, y2, v, frame_rows: int, r1=None) -> dict:
        """Outputs of the three sites where y1 and y2 are the branches' outputs; the last site starts from r1 if given."""
        f = acid.acid_norm_site_forward
        u1 = f(x, branch_dtype=torch.bfloat16, want_r=False, **self._first(v, frame_rows))[1]
        out = dict(u1=u1)
        out["r1"], out["u2"] = f(x, y1, **self._middle(v, frame_rows))
        out["r2"] = f(out["r1"] if r1 is None else r1, y2, want_u=False, **self._last(v, frame_rows))[0]
        return out

    def forward(self, x: torch.Tensor, temb: torch.Tensor, frame_rows: int, keep: bool = False):
        """r2 [rows, d] (fp32) from x [rows, d] (fp32) and temb [frames, d]; with ``keep`` also the dict of u1, y1,
        r1, u2, y2, r2."""
        v = self.vectors(self.modulation(temb))
        f = acid.acid_norm_site_forward
        _, u1 = f(x, branch_dtype=torch.bfloat16, want_r=False, **self._first(v, frame_rows))
        y1 = self.attention(u1)
        r1, u2 = f(x, y1, **self._middle(v, frame_rows))
        y2 = self.mlp(u2)
        r2, _ = f(r1, y2, want_u=False, **self._last(v, frame_rows))
        return (r2, dict(u1=u1, y1=y1, r1=r1, u2=u2, y2=y2, r2=r2)) if keep else r2

    def site_errors(self, x, temb, frame_rows: int, seen: dict):
        """(loss, errors, vectors): the sites' outputs less those of ``seen`` (a full-precision forward's dict), each
        site on seen's inputs, and half their squares' sum over rows."""
        v = self.vectors(self.modulation(temb))
        got = self.sites(x, seen["y1"], seen["y2"], v, frame_rows, r1=seen["r1"])
        errors = {n: got[n].float() - seen[n].float() for n in ("u1", "r1", "u2", "r2")}
        loss = sum(0.5 * e.square().sum() for e in errors.values()) / x.shape[0]
        return loss, errors, (v, got)

    def gradients(self, x, temb, frame_rows: int, seen: dict):
        """(loss, dtemb, db_mod) of site_errors' loss."""
        loss, errors, (v, got) = self.site_errors(x, temb, frame_rows, seen)
        e = {n: t / x.shape[0] for n, t in errors.items()}
        b = acid.acid_norm_site_backward
        first = b(e["u1"], x, **self._first(v, frame_rows))
        middle = b(e["u2"].bfloat16(), got["r1"], seen["y1"], dr=e["r1"], **self._middle(v, frame_rows))
        last = b(None, None, seen["y2"], dr=e["r2"], **self._last(v, frame_rows))
        dmod = torch.cat([first["dshift"], first["dscale"], middle["dgate"], middle["dshift"], middle["dscale"],
                          last["dgate"]], 1)
        dtemb, dbias = acid.acid_q4_linear_backward(dmod, self.mod_q4, temb, silu=True)
        return loss, dtemb, dbias

    def calibrate(self, x, temb, frame_rows: int, seen: dict, steps: int = 20, rate: float = 0.5) -> list[float]:
        """Moves mod_b against the gradient, ``steps`` times; the loss at the start and after each step.  Along a bias
        column the loss curves by about 1 where the rows' normed values differ, and by more where they agree (a branch's
        output that hardly changes from row to row), so a step that raises the loss is taken back and the rate halved."""
        loss, _, dbias = self.gradients(x, temb, frame_rows, seen)
        losses = [float(loss)]
        for _ in range(steps):
            before = self.mod_b.clone()
            self.mod_b -= rate * dbias
            loss, _, moved = self.gradients(x, temb, frame_rows, seen)
            if float(loss) < losses[-1]:
                losses.append(float(loss))
                dbias = moved
            else:
                losses.append(losses[-1])
                self.mod_b.copy_(before)
                rate /= 2
        return losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--d", type=int, default=1536)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--hidden", type=int, default=None, help="of the MLP (default 4 d)")
    ap.add_argument("--frames", type=int, default=21)
    ap.add_argument("--tokens", type=int, default=390, help="rows of a frame")
    ap.add_argument("--group", type=int, default=64, choices=(32, 64, 128))
    ap.add_argument("--zeros", action="store_true", help="zero points beside the scales")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    weights = random_weights(a.d, a.hidden or 4 * a.d, a.seed)
    gen = torch.Generator(device="cuda").manual_seed(a.seed + 1)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", dtype=torch.float32, generator=gen)

    x = normal(a.frames * a.tokens, a.d)
    # embeddings of neighbouring timesteps: a common part, and a tenth of its size of their own
    temb = normal(1, a.d) + 0.1 * normal(a.frames, a.d)
    full = AdaLNBlock(weights, a.heads, group=None)
    want, seen = full.forward(x, temb, a.tokens, keep=True)
    block = AdaLNBlock(weights, a.heads, a.group, a.zeros)

    def error():
        return float((block.forward(x, temb, a.tokens) - want).norm() / (want - x).norm())

    before = error()
    losses = block.calibrate(x, temb, a.tokens, seen, a.steps)
    print(json.dumps({"rows": x.shape[0], "d": a.d, "group": a.group, "zeros": a.zeros, "error": before,
                      "calibrated": error(), "loss": losses[0], "calibrated_loss": losses[-1]}))


if __name__ == "__main__":
    main()
