"""The layer step that runs the experts' operators together (a routing step's
rows through the experts, the combine and all gradients; the same experts in 4
bits), call by call against the oracle in 64 bits."""
import dataclasses

import numpy as np
import pytest
import torch

import expert_cases as C
import oracle
import oracle.experts as X
from paper_2609_36959_amd import binding as B
from paper_2609_36959_amd import experts as M
from paper_2609_36959_amd import pipeline as PL
from paper_2609_36959_amd import workload as W

pytestmark = pytest.mark.gpu

F = 96


@pytest.fixture(scope="module")
def step():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    w = dataclasses.replace(W.WORKLOADS["tiny"], T=512, d=320)
    s = M.ExpertStep(w, seed=0, f=F, device="cuda:0", route_device="cpu")
    yield s
    torch.cuda.synchronize()
    s.close()
    torch.cuda.empty_cache()


def near(t, want, slack, what):
    C.close(C.host(t), want, slack, what)


def test_training_step(step):
    w = step.w
    step.forward()
    topk, pos = step.topk.cpu().numpy(), step.pos.cpu().numpy()
    rows, _, off = X.group(topk, pos, w.E)
    assert np.array_equal(step.rows.cpu().numpy(), rows)
    assert np.array_equal(step.expert_offsets.cpu().numpy(), off)
    assert torch.equal(step.packed[step.pos.long()],
                       step.x[:, None].expand(-1, w.K, -1))
    w_in, w_down = C.host(step.w_in), C.host(step.w_down)
    a = C.host(step.packed)[rows]
    gu, e_gu, h, e_h = C.gate_up(a, off, w_in, step.act)
    near(step.gate_up, gu, e_gu, "gate_up")
    near(step.h, h, e_h, "h")
    kept_gu, kept_h = C.host(step.gate_up), C.host(step.h)
    y, size = X.per_expert(kept_h, off, w_down)
    near(step.eo[step.rows.long()], y, C.BF16 * np.abs(y) + 1.01 * C.product_bound(F, size), "eo")
    want, _ = oracle.combine(PL.bf16_bits(step.eo), pos, step.gates.cpu().numpy())
    assert np.array_equal(PL.bf16_bits(step.y), want)

    dy = C.dev(C.bf16(np.random.default_rng(5), w.T, w.d))
    step.backward(dy)
    g, v = step.gates.cpu().numpy().astype(np.float64), C.host(dy)
    deo = g[:, :, None] * v[:, None]
    near(step.deo[step.pos.long()], deo, C.BF16 * np.abs(deo), "dexpert_out")
    eo = C.host(step.eo)[pos]
    terms = v[:, None] * eo
    near(step.dgates, terms.sum(2), C.product_bound(w.d, np.abs(terms).sum(2)), "dgates")
    dout = C.host(step.deo)[rows]
    near(step.gate_up, *C.down_gradient(dout, off, w_down, kept_gu, step.act), "dgate_up")
    most = int(np.diff(off).max())
    for t, p, q in ((step.dw_down, dout, kept_h), (step.dw_in, C.host(step.gate_up), a)):
        d, size = X.outer_sums(p, q, off)
        near(t, d, C.BF16 * np.abs(d) + 1.01 * C.product_bound(most, size), "weight gradient")
    d, size = X.per_expert(C.host(step.gate_up), off, w_in.transpose(0, 2, 1))
    near(step.dpacked[step.rows.long()], d,
         C.BF16 * np.abs(d) + 1.01 * C.product_bound(2 * F, size), "dpacked")
    want, _ = oracle.combine(PL.bf16_bits(step.dpacked), pos, np.ones_like(g, np.float32))
    assert np.array_equal(PL.bf16_bits(step.dx), want)


def test_serving_in_four_bits(step):
    w = step.w
    serve = M.MxExperts(step.w_in, step.w_down, w.T, w.K)
    value = lambda c: X.dequantize(*(t.cpu().numpy() for t in c))  # noqa: E731
    w_in, w_down = value(serve.w_in), value(serve.w_down)
    for T, drop in ((w.T, False), (7, True), (1, False)):
        x, topk, gates = step.x[:T], step.topk[:T].clone(), step.gates[:T].contiguous()
        y = torch.full_like(x, float("nan"))
        pos = None
        if drop:
            topk[3, 1], topk[5, 0] = -1, w.E
            pos = serve.pos[:T].clone()
            pos[3, 1] = pos[5, 0] = -1
        serve.run(x, topk, gates, y, pos)
        rows, tokens, off = X.group(topk.cpu().numpy(), None, w.E)
        n = int(off[-1])
        assert np.array_equal(serve.rows[:n].cpu().numpy(), rows[:n])
        xq = [t[:T] for t in serve.x]
        codes, scales = X.quantize(C.host(x))
        assert np.array_equal(xq[0].cpu().numpy(), codes)
        assert np.array_equal(xq[1].cpu().numpy(), scales)
        _, _, h, e_h = C.gate_up(value(xq)[tokens[:n]], off, w_in, B.ACT_SILU)
        near(serve.h[:n], h, e_h, "h")
        out, size = X.per_expert(value([t[:n] for t in serve.hq]), off, w_down)
        at = torch.from_numpy(rows[:n]).long().cuda()
        near(serve.out[at], out, C.BF16 * np.abs(out) + 1.01 * C.product_bound(F, size), "out")
        p = (serve.pos[:T] if pos is None else pos).cpu().numpy()
        want, _ = oracle.combine(PL.bf16_bits(serve.out[:T * w.K]), p, gates.cpu().numpy())
        assert np.array_equal(PL.bf16_bits(y), want)


def test_captured_in_a_graph(step):
    """A captured step gives the eager step's outputs on every replay, with
    eager work between the replays, and follows its inputs' values."""
    dy = C.dev(C.bf16(np.random.default_rng(6), step.w.T, step.w.d))
    serve = M.MxExperts(step.w_in, step.w_down, step.w.T, step.w.K)
    y4 = torch.empty_like(step.y)

    def run():
        step.forward()
        step.backward(dy)
        serve.run(step.x, step.topk, step.gates, y4)
        return [step.y, step.dx, step.dgates, step.dw_in, step.dw_down, y4]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for i in range(4):
        step.x.mul_(0.5 if i % 2 else 2.0)
        want = [t.clone() for t in run()]
        for t in outs:
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(want, outs):
            assert torch.equal(p, q)


def test_command(capsys):
    M.main(["--workload", "tiny", "--width", "64", "--steps", "2"])
    said = capsys.readouterr().out
    assert "training step" in said and "4-bit serving" in said
