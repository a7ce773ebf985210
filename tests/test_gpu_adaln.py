"""The block that runs the norm sites and the 4-bit modulation together, and its calibration.

Tolerances.  A branch passes its value through six roundings to bf16 one behind the other (the site's output, the
first product, what is between, the second product), each at most 2^-8 of an element: 2.5e-2 of the branches'
share r2 - x.  A directional derivative along the gradient: the errors carry the rounding of two bf16 outputs, up to
2^-8 of values of size 1 beside errors of 0.01 and more, a quarter of each, and 111 x 256 of them of either sign enter
the sum, a quarter / sqrt(28416) = 0.2%; rounding the site's gradients to bf16 0.4%; 1% in all."""

import json

import numpy as np
import pytest

import oracle.adaln_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
D, HEADS, HIDDEN, FRAMES, TOKENS = 256, 2, 512, 3, 37


@pytest.fixture(autouse=True)
def fp32_by_default():
    """Whatever default another module of the run has set."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.fixture(scope="module")
def adaln():
    import __graft_entry__ as g

    g.build()
    from paper_2607_12358_gb300 import adaln as a

    return a


def f64(t):
    return t.double().cpu().numpy()


def inputs(adaln):
    w = adaln.random_weights(D, HIDDEN, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    normal = lambda *s: torch.randn(*s, device="cuda", dtype=torch.float32, generator=gen)  # noqa: E731
    x = normal(FRAMES * TOKENS, D)
    temb = normal(1, D) + 0.1 * normal(FRAMES, D)
    return w, x, temb


def mod_values(adaln, block):
    """The modulation's weight as the block holds it, in 64 bits."""
    if block.mod_q4 is None:
        return f64(block.w["mod_w"])
    return f64(adaln.acid.acid_q4_dequantize(block.mod_q4))


def modulation(mod_w, mod_b, temb):
    return temb / (1 + np.exp(-temb)) @ mod_w.T + mod_b


def sites(w, mod, x, y1, y2, r1=None):
    v = [mod[:, i * D:(i + 1) * D] for i in range(6)]
    _, u1 = O.norm_site(x, None, shift=v[0], scale=v[1], post_norm="none", group_rows=TOKENS)
    out = dict(u1=u1)
    if y1 is not None:
        out["r1"], out["u2"] = O.norm_site(x, y1, gate=v[2], shift=v[3], scale=v[4], post_w=f64(w["w1"]), group_rows=TOKENS)
    if y2 is not None:
        out["r2"], _ = O.norm_site(out["r1"] if r1 is None else r1, y2, gate=v[5], post_w=f64(w["w2"]), pre_norm="none",
                                   group_rows=TOKENS)
    return out


def linear(w, name, a):
    return a @ f64(w[name]).T + f64(w[name + "_b"])


@pytest.mark.parametrize("group,zeros", [(None, False), (64, True), (32, False)])
def test_forward_is_the_definition(adaln, group, zeros):
    w, x, temb = inputs(adaln)
    block = adaln.AdaLNBlock(w, HEADS, group, zeros)
    got = block.forward(x, temb, TOKENS)
    mod = modulation(mod_values(adaln, block), f64(block.mod_b), f64(temb))
    np.testing.assert_allclose(f64(block.modulation(temb)), mod, rtol=0, atol=1e-5)
    nx = f64(x)
    qkv = linear(w, "qkv", sites(w, mod, nx, None, None)["u1"])
    a = np.empty((len(nx), D))
    for h in range(HEADS):
        q, k, v = (qkv[:, i * D:(i + 1) * D][:, h * 128:(h + 1) * 128] for i in range(3))
        s = q @ k.T / np.sqrt(128)
        p = np.exp(s - s.max(-1, keepdims=True))
        a[:, h * 128:(h + 1) * 128] = p @ v / p.sum(-1, keepdims=True)
    y1 = linear(w, "out", a)
    u2 = sites(w, mod, nx, y1, None)["u2"]
    h = linear(w, "fc1", u2)
    h = 0.5 * h * (1 + np.tanh(np.sqrt(2 / np.pi) * (h + 0.044715 * h ** 3)))
    want = sites(w, mod, nx, y1, linear(w, "fc2", h))["r2"]
    assert np.linalg.norm(f64(got) - want) <= 2.5e-2 * np.linalg.norm(want - nx)


def test_gradients_against_differences(adaln):
    w, x, temb = inputs(adaln)
    _, seen = adaln.AdaLNBlock(w, HEADS, None).forward(x, temb, TOKENS, keep=True)
    block = adaln.AdaLNBlock(w, HEADS, 128, False)
    loss, dtemb, dbias = block.gradients(x, temb, TOKENS, seen)
    mod_w, bias, nt, nx = mod_values(adaln, block), f64(block.mod_b), f64(temb), f64(x)
    ns = {k: f64(v) for k, v in seen.items()}

    def exact(b, t):
        got = sites(w, modulation(mod_w, b, t), nx, ns["y1"], ns["y2"], ns["r1"])
        return sum(0.5 * ((got[n] - ns[n]) ** 2).sum() for n in ("u1", "r1", "u2", "r2")) / len(nx)

    for grad, moved in ((f64(dbias), lambda v: exact(bias + v, nt)), (f64(dtemb), lambda v: exact(bias, nt + v))):
        size = np.linalg.norm(grad)
        step = 1e-4 * grad / size
        slope = (moved(step) - moved(-step)) / 2e-4
        assert abs(slope - size) <= 0.01 * size


def test_calibration_lowers_the_error(adaln):
    w, x, temb = inputs(adaln)
    want, seen = adaln.AdaLNBlock(w, HEADS, None).forward(x, temb, TOKENS, keep=True)
    block = adaln.AdaLNBlock(w, HEADS, 64, True)
    before = (block.forward(x, temb, TOKENS) - want).norm()
    losses = block.calibrate(x, temb, TOKENS, seen, steps=20)
    assert len(losses) == 21 and losses[-1] < 0.5 * losses[0]
    assert (block.forward(x, temb, TOKENS) - want).norm() < before
    assert not torch.equal(block.mod_b, w["mod_b"])  # the block's own copy


def test_command(adaln, capsys):
    adaln.main(["--d", "256", "--heads", "2", "--frames", "3", "--tokens", "37", "--group", "32", "--steps", "5"])
    out = json.loads(capsys.readouterr().out)
    assert out["rows"] == 111 and out["calibrated_loss"] < out["loss"] and out["calibrated"] < out["error"]
