"""Gradients of the combine against the formula in 64 bits, and of the whole
pass against differences."""
import numpy as np
import pytest
import torch

import expert_cases as C
import oracle.experts as X
from paper_2609_36959_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    B.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def inputs(T, K, d, drop, seed=0):
    rng = np.random.default_rng([seed, T, K, d])
    pos = rng.permutation(T * K).astype(np.int32).reshape(T, K)
    gone = rng.random((T, K)) < drop
    pos[gone] = rng.choice([-1, T * K, 2**31 - 1, -2**31], gone.sum())
    gates = rng.standard_normal((T, K)).astype(np.float32)
    eo = C.bf16(rng, T * K, d)
    eo[np.setdiff1d(np.arange(T * K), pos)] = 0x7fc0
    return C.bf16(rng, T, d), eo, pos, gates


@pytest.mark.parametrize("T,K,d,drop", [
    (1, 1, 8, 0), (1, 16, 24, 0), (5, 3, 1032, 0.3), (130, 8, 512, 0.02), (33, 6, 2048, 0),
    (7, 10, 7168, 0.2), (3, 2, 40000, 0), (1000, 2, 64, 1.0)])
def test_gradients(T, K, d, drop):
    dy, eo, pos, gates = inputs(T, K, d, drop)
    mark = np.full((T * K, d), 0x4123, np.uint16)
    deo, dg = C.dev(mark), torch.full((T, K), float("nan"), device="cuda")
    args = (C.dev(dy), C.dev(eo), C.dev(pos), C.dev(gates))
    B.cobalt_combine_backward(*args, deo, dg)
    vy, ve = X.wide(dy), X.wide(eo)
    want_g, slack_g = np.zeros((2, T, K))
    got, hit = C.host(deo), np.zeros(T * K, bool)
    for t in range(T):
        for j in range(K):
            p = pos[t, j]
            if not 0 <= p < T * K:
                continue
            hit[p] = True
            want = np.float64(gates[t, j]) * vy[t]
            C.close(got[p], want, (C.BF16 + 2.0 ** -23) * np.abs(want), f"row {p}")
            terms = vy[t] * ve[p]
            want_g[t, j], slack_g[t, j] = terms.sum(), C.product_bound(d, np.abs(terms).sum())
    C.close(C.host(dg), want_g, slack_g + 2.0 ** -23 * np.abs(want_g), "dgates")
    assert (deo.view(torch.int16).cpu().numpy()[~hit] == 0x4123).all()
    # either alone, and the gradient in the rows' place
    one, two = C.dev(mark), torch.empty_like(dg)
    B.cobalt_combine_backward(args[0], None, args[2], args[3], one)
    B.cobalt_combine_backward(args[0], args[1], args[2], None, None, two)
    rows = C.dev(eo)
    three = torch.empty_like(dg)
    B.cobalt_combine_backward(args[0], rows, args[2], args[3], rows, three)
    bits = lambda t: t.view(torch.int16)  # noqa: E731
    assert torch.equal(bits(one), bits(deo))
    assert torch.equal(bits(rows)[torch.from_numpy(hit).cuda()],
                       bits(deo)[torch.from_numpy(hit).cuda()])
    assert torch.equal(two.view(torch.int32), dg.view(torch.int32))
    assert torch.equal(three.view(torch.int32), dg.view(torch.int32))


def test_launches_over_token_ranges(monkeypatch):
    dy, eo, pos, gates = inputs(300, 4, 136, 0.1)
    args = [C.dev(a) for a in (dy, eo, pos, gates)]
    a = [C.dev(np.zeros_like(eo)), torch.empty(300, 4, device="cuda")]
    b = [C.dev(np.zeros_like(eo)), torch.empty(300, 4, device="cuda")]
    B.cobalt_combine_backward(*args, *a)
    monkeypatch.setenv("COBALT_MAX_LAUNCH_ITEMS", "4096")
    B.cobalt_combine_backward(*args, *b)
    assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1], b[1])


def test_gate_gradient_against_differences():
    """A loss sum(c * y) of the combine with fp32 sums: its change with a gate
    is exact to the sums' rounding, since y is linear in the gates."""
    T, K, d = 6, 3, 256
    dy, eo, pos, gates = inputs(T, K, d, 0)
    dg = torch.empty(T, K, device="cuda")
    B.cobalt_combine_backward(C.dev(dy), C.dev(eo), C.dev(pos), None, None, dg)

    def loss(g):
        y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        y32 = torch.empty(T, d, device="cuda")
        B.cobalt_combine(C.dev(eo), C.dev(pos), C.dev(g.astype(np.float32)), y, y32)
        return (X.wide(dy) * C.host(y32)).sum()

    for t in range(T):
        for j in range(K):
            up, down = gates.copy(), gates.copy()
            up[t, j] += 0.5
            down[t, j] -= 0.5
            step = float(up[t, j]) - float(down[t, j])
            num = (loss(up) - loss(down)) / step
            # each y32 is off by K roundings of sums under 16 on |dy| < 6
            assert abs(num - float(dg[t, j])) < 2 * d * 6 * K * 16 * 2.0 ** -24
