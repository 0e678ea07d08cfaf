"""The experts' operators where their tiles differ: sizes at which a call takes
each of its tiles' shapes, streams the weights or splits an expert's rows, more
experts than one wave looks through, launches over ranges; and the gradients
against differences of the 64-bit forward pass."""
import numpy as np
import pytest
import torch

import expert_cases as C
import oracle.experts as X
import test_gpu_experts as G
import test_gpu_mx as Q
from paper_2609_36959_amd import binding as B

pytestmark = pytest.mark.gpu
gpu = G.gpu


def spread(M, E, seed=0):
    """M rows over E experts, some twice as popular."""
    p = 1.0 + np.arange(E) % 2
    return [int(v) for v in np.random.default_rng(seed).multinomial(M, p / p.sum())]


# (rows of each expert, places behind, d, f). All have sizes that fill no tile.
CASES = [
    (spread(7284, 3), 5, 1672, 40),      # few columns, many rows of few experts
    ([11201, 0], 0, 88, 1136),           # one expert has all; long sums over rows
    (spread(6813, 5), 1, 1160, 40),
    ([19001], 0, 40, 72),
    (spread(2173, 1), 3, 72, 904),
    ([4247], 0, 8, 808),
    (spread(300, 20), 0, 264, 1576),     # a handful of rows each, wide
    (spread(300, 300), 2, 520, 72),      # more experts than lanes times four
    (spread(211, 20), 0, 3176, 16),
    (spread(8000, 1), 0, 2056, 104),
]
MX_CASES = [
    ([4247], 0, 96, 832),
    (spread(3137, 3), 7, 64, 1184),
    (spread(6850, 2), 0, 992, 32),
    (spread(6813, 5), 2, 1152, 96),
    (spread(300, 300), 2, 544, 64),
]


def name(case):
    counts, _, d, f = case
    return f"{sum(counts)}rows-{len(counts)}x-d{d}-f{f}"


@pytest.mark.parametrize("case", CASES, ids=name)
def test_forward(case):
    G.test_forward(case, B.ACT_SILU)


@pytest.mark.parametrize("case", CASES, ids=name)
def test_backward(case):
    G.test_backward(case, B.ACT_GELU)


@pytest.mark.parametrize("case", MX_CASES, ids=name)
def test_mx(case):
    Q.test_products(case, B.ACT_SILU)


def test_split_rows_need_a_workspace():
    """Rows of few experts with small weights are summed in parts, the parts in
    fp32 in the workspace; other sizes need none to speak of."""
    size = B.cobalt_expert_backward_workspace_bytes
    assert size(16384, 4, 512, 256) >= 2 * 4 * 512 * 512 * 4
    assert size(16384, 64, 2048, 1024) == size(100, 4, 512, 256) == 256


def run_all(b, x_codes, w_codes):
    """Every output of the calls over tiles or blocks of rows."""
    h, gu, out = G.run_forward(b, B.ACT_SILU)
    B.cobalt_expert_down(h, b.t_off, C.dev(b.w_down), b.t_rows, out)
    ws = B.expert_backward_workspace_for(b.M, b.E, b.d, b.f)
    dgu, dx, dw, dwi = (G.marked(b.M, 2 * b.f), G.marked(b.n, b.d), G.marked(b.E, b.d, b.f),
                        G.marked(b.E, 2 * b.f, b.d))
    dout = C.dev(b.x)
    B.cobalt_expert_down_backward(dout, b.t_rows, b.t_off, C.dev(b.w_down), gu, h, dgu, dw, ws)
    B.cobalt_expert_gate_up_backward(dgu, C.dev(b.x), b.t_rows, b.t_off, C.dev(b.w_in), dx, dwi, ws)
    mh, back = G.marked(b.M, b.f), G.marked(b.n, b.d)
    B.cobalt_mx_quantize(C.dev(b.x), *x_codes)
    B.cobalt_mx_quantize(C.dev(b.w_in), *w_codes)
    B.cobalt_mx_gate_up(*x_codes, b.t_rows, b.t_off, *w_codes, mh)
    B.cobalt_mx_dequantize(*x_codes, back)
    return [h, gu, out, dgu, dx, dw, dwi, mh, back]


@pytest.mark.parametrize("case", [([40, 0, 700], 1, 544, 288), ([1200, 1100], 0, 96, 64),
                                  ([1, 2, 1], 0, 1056, 96)], ids=name)
def test_launches_over_ranges(case, monkeypatch):
    b = G.Block(case)
    codes = lambda *s: (Q.u8(*s[:-1], s[-1] // 2), Q.u8(*s[:-1], s[-1] // 32))  # noqa: E731
    xc, wc = codes(b.n, b.d), codes(b.E, 2 * b.f, b.d)
    whole = run_all(b, xc, wc)
    kept = [t.clone() for t in (*xc, *wc)]
    monkeypatch.setenv("COBALT_MAX_LAUNCH_ITEMS", "4096")
    for t in (*xc, *wc):
        t.fill_(0xA5)
    for p, q in zip(whole + kept, run_all(b, xc, wc) + [*xc, *wc]):
        assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("kind", [B.ACT_SILU, B.ACT_GELU])
def test_gradients_against_differences(kind):
    """A loss sum(c * out) of the 64-bit forward pass changes along a direction
    as the gradients say. The bounds hold what the bf16 between the calls adds:
    g, u, h and dgate_up are rounded once (2^-8 of each at most), and a'(g)
    moves with g by |g a''(g)| 2^-8, |g a''| being under 2; fp32 sums add less
    than a tenth of that, the differences themselves about 1e-8."""
    b = G.Block(([5, 9], 0, 40, 24), rows=False)
    x, w_in, w_down = X.wide(b.x), X.wide(b.w_in), X.wide(b.w_down)
    cb = C.bf16(b.rng, b.M, b.d)
    c = X.wide(cb)
    h, gu, _ = G.run_forward(b, kind)
    ws = B.expert_backward_workspace_for(b.M, b.E, b.d, b.f)
    dgu, dx = G.marked(b.M, 2 * b.f), G.marked(b.M, b.d)
    dw_down = torch.empty(b.E, b.d, b.f, device="cuda")
    dw_in = torch.empty(b.E, 2 * b.f, b.d, device="cuda")
    B.cobalt_expert_down_backward(C.dev(cb), None, b.t_off, C.dev(b.w_down), gu, h, dgu, dw_down,
                                  ws, act=kind, flags=B.GRAD_FLOAT)
    B.cobalt_expert_gate_up_backward(dgu, C.dev(b.x), None, b.t_off, C.dev(b.w_in), dx, dw_in, ws,
                                     flags=B.GRAD_FLOAT)

    def loss(x, w_in, w_down):
        gu, _ = X.per_expert(x, b.off, w_in)
        h = X.act(gu[:, :b.f], kind) * gu[:, b.f:]
        return float((c * X.per_expert(h, b.off, w_down)[0]).sum())

    v, _ = X.per_expert(x, b.off, w_in)
    g, u = v[:, :b.f], v[:, b.f:]
    dh = np.abs(X.per_expert(c, b.off, w_down.transpose(0, 2, 1))[0])
    a = np.abs(X.act(g, kind))
    e = C.BF16 * np.concatenate([dh * np.abs(u) * (2 * np.abs(X.act_slope(g, kind)) + 2),
                                 dh * (1.13 * np.abs(g) + a)], 1)
    eps = 1e-4
    for part, grad in (("x", dx), ("w_in", dw_in), ("w_down", dw_down)):
        args = {"x": x, "w_in": w_in, "w_down": w_down}
        to = b.rng.standard_normal(args[part].shape)
        up, down = dict(args), dict(args)
        up[part], down[part] = args[part] + eps * to, args[part] - eps * to
        want = (loss(**up) - loss(**down)) / (2 * eps)
        got = C.host(grad)
        if part == "x":
            off = (e * np.abs(X.per_expert(to, b.off, w_in)[0])).sum()
        elif part == "w_in":
            off = (e * np.abs(X.per_expert(x, b.off, to)[0])).sum()
        else:
            off = C.BF16 * (np.abs(c) * X.per_expert(a * np.abs(u), b.off, np.abs(to))[0]).sum()
        off = 1.1 * off + C.BF16 * np.abs(got * to).sum() + 1e-6 * np.abs(got).sum()
        assert abs((got * to).sum() - want) <= off, part
