"""The experts' bf16 products, their gradients and the grouping of pairs,
through the public calls, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import expert_cases as C
import oracle.experts as X
from paper_2609_36959_amd import binding as B

pytestmark = pytest.mark.gpu

MARK = 0x4123  # bf16 bits of 10.1875 in places that no call may write


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    B.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def marked(*shape):
    return C.dev(np.full(shape, MARK, np.uint16))


# ---------------------------------------------------------------- grouping
@pytest.mark.parametrize("T,K,E,drop,with_pos", [
    (1, 1, 1, 0, False), (1, 8, 64, 0, False), (63, 2, 5, 0.3, True), (1000, 6, 64, 0, True),
    (1025, 8, 3, 0.9, True), (4099, 2, 4096, 0.1, False), (4097, 16, 256, 0, True),
    (70001, 3, 7, 0.01, True), (40000, 8, 2049, 0, True), (50, 4, 10, 1.0, True)])
def test_group(T, K, E, drop, with_pos):
    rng = np.random.default_rng(T)
    topk = rng.integers(0, E, (T, K)).astype(np.int32)
    gone = rng.random((T, K)) < drop
    topk[gone] = rng.choice([-1, E, 2**31 - 1, -2**31], gone.sum())
    pos = rng.permutation(T * K).astype(np.int32).reshape(T, K) if with_pos else None
    key = np.where((topk < 0) | (topk >= E), E, topk).reshape(-1)
    order = np.argsort(key, kind="stable")
    off = np.searchsorted(key[order], np.arange(E + 1))
    n = off[E]
    rows = np.full(T * K, -1)
    rows[:n] = (order if pos is None else pos.reshape(-1)[order])[:n]
    tokens = np.full(T * K, -1)
    tokens[:n] = order[:n] // K
    ws = B.expert_group_workspace_for(T, K, E)
    ws.fill_(0x5A)
    got = [torch.full((m,), 77, dtype=torch.int32, device="cuda") for m in (T * K, T * K, E + 1)]
    B.cobalt_expert_group(C.dev(topk), C.dev(pos), E, got[0], got[2], ws, tokens=got[1])
    for g, w in zip(got, (rows, tokens, off)):
        assert np.array_equal(g.cpu().numpy(), w)
    got[0].fill_(77)
    B.cobalt_expert_group(C.dev(topk), C.dev(pos), E, got[0], got[2], ws)
    assert np.array_equal(got[0].cpu().numpy(), rows)


def test_group_of_no_tokens():
    off = torch.full((9,), 5, dtype=torch.int32, device="cuda")
    none = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    B.cobalt_expert_group(none, None, 8, none.view(-1), off, B.expert_group_workspace_for(0, 2, 8))
    assert not off.any()


# ---------------------------------------------------------------- products
# (rows of each expert, places behind the last expert, d, f): one row; widths
# under, at and over the tiles; experts without rows, at the ends too; few rows
# and many; counts that fill tiles exactly and by one more or less
CASES = [
    ([1], 0, 8, 8),
    ([0, 1, 0], 2, 24, 40),
    ([3, 0, 17, 1], 0, 136, 72),
    ([16, 15, 33], 1, 264, 128),
    ([1] * 70, 0, 64, 32),
    ([64, 65, 63, 0, 128], 5, 512, 256),
    ([256, 257], 0, 320, 192),
    ([0, 700, 41], 3, 200, 520),
    ([300, 260, 5, 511], 0, 1032, 264),
    ([2, 1, 3, 0, 1], 1, 2056, 1000),
]
IDS = [f"{sum(c)}rows-{len(c)}x-d{d}-f{f}" for c, _, d, f in CASES]


class Block:
    """An expert block of a case: inputs as bits and as float64. Rows are
    taken from a larger buffer in random order; `hole` of the places name no
    row. Buffer rows without a place hold NaN."""

    def __init__(self, case, seed=0, rows=True, hole=0.0, scale=1.0):
        counts, behind, d, f = case
        rng = np.random.default_rng([seed, d, f])
        self.rng, self.d, self.f, self.E = rng, d, f, len(counts)
        self.off = C.offsets_of(counts)
        self.used = int(self.off[-1])
        self.M = self.used + behind
        self.n = self.M + 3 if rows else self.M
        self.rows = rng.permutation(self.n)[:self.M].astype(np.int32) if rows else None
        self.x = C.bf16(rng, self.n, d, scale=scale)
        if rows:
            self.rows[self.used:] = -1
            gone = rng.random(self.M) < hole
            self.rows[gone] = rng.choice([-1, self.n, 2**31 - 1, -2**31], gone.sum())
            lone = np.setdiff1d(np.arange(self.n), self.rows)
        else:
            lone = np.arange(self.used, self.M)
        self.lone = lone
        self.x[lone] = 0x7fc0
        self.w_in = C.bf16(rng, self.E, 2 * f, d, scale=d ** -0.5)
        self.w_down = C.bf16(rng, self.E, d, f, scale=f ** -0.5)
        self.t_rows, self.t_off = C.dev(self.rows), C.dev(self.off)

    def places(self, bits):
        """Float64 rows of a row buffer at the places that belong to an expert."""
        v = X.wide(bits)
        v[self.lone] = 0
        a = X.taken(v, self.rows, self.M)
        a[self.used:] = 0
        return a

    def scattered(self, y, slack):
        """The row buffer that a call writes, and its bound; -1 = not written."""
        out, b = np.zeros((2, self.n, y.shape[1]))
        hit = np.zeros(self.n, bool)
        for i in range(self.used):
            r = i if self.rows is None else self.rows[i]
            if 0 <= r < self.n:
                out[r], b[r], hit[r] = y[i], slack[i], True
        return out, b, hit


def check_rows(t, want, slack, hit, what):
    C.close(C.host(t)[hit], want[hit], slack[hit], what)
    rest = t.cpu().view(torch.int16).numpy().view(np.uint16)[~hit]
    assert (rest == MARK).all(), f"{what}: wrote a row that no place names"


def run_forward(b, kind, keep=True):
    h, gu = marked(b.M, b.f), marked(b.M, 2 * b.f)
    out = marked(b.n, b.d)
    B.cobalt_expert_gate_up(C.dev(b.x), b.t_rows, b.t_off, C.dev(b.w_in), h, gu if keep else None,
                            act=kind)
    return h, gu, out


@pytest.mark.parametrize("kind", [B.ACT_SILU, B.ACT_GELU])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case, kind):
    for rows, hole in ((True, 0.0), (True, 0.2), (False, 0.0)):
        b = Block(case, rows=rows, hole=hole)
        h, gu, out = run_forward(b, kind)
        place = np.arange(b.M) < b.used
        want_gu, e_gu, want_h, e_h = C.gate_up(b.places(b.x), b.off, X.wide(b.w_in), kind)
        check_rows(gu, want_gu, e_gu, place, "gate_up")
        check_rows(h, want_h, e_h, place, "h")
        again, _, _ = run_forward(b, kind, keep=False)
        assert torch.equal(again.view(torch.int16), h.view(torch.int16))
        B.cobalt_expert_down(h, b.t_off, C.dev(b.w_down), b.t_rows, out)
        a = C.host(h)
        a[b.used:] = 0
        y, size = X.per_expert(a, b.off, X.wide(b.w_down))
        check_rows(out, *b.scattered(y, C.BF16 * np.abs(y) + 1.01 * C.product_bound(b.f, size)),
                   "out")


@pytest.mark.parametrize("kind", [B.ACT_SILU, B.ACT_GELU])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case, kind):
    for rows, hole in ((True, 0.2), (False, 0.0)):
        b = Block(case, rows=rows, hole=hole)
        gu, h = C.bf16(b.rng, b.M, 2 * b.f), C.bf16(b.rng, b.M, b.f)
        gu[b.used:], h[b.used:] = 0x7fc0, 0x7f80
        dout = C.bf16(b.rng, b.n, b.d, scale=0.1)
        dout[b.lone] = 0x7fc0
        ws = B.expert_backward_workspace_for(b.M, b.E, b.d, b.f)
        place = np.arange(b.M) < b.used

        dgu = marked(b.M, 2 * b.f)
        dw = marked(b.E, b.d, b.f)
        B.cobalt_expert_down_backward(C.dev(dout), b.t_rows, b.t_off, C.dev(b.w_down), C.dev(gu),
                                      C.dev(h), dgu, dw, ws, act=kind)
        v = X.wide(gu)
        v[b.used:] = 0
        check_rows(dgu, *C.down_gradient(b.places(dout), b.off, X.wide(b.w_down), v, kind), place,
                   "dgate_up")
        hv = X.wide(h)
        hv[b.used:] = 0
        most = max(case[0])

        def check_dw(t, a, c, add=0.0, f32=False):
            y, size = X.outer_sums(a, c, b.off)
            slack = 1.01 * C.product_bound(most, size)
            slack = slack + (2.0 ** -23 * (np.abs(y) + np.abs(add)) if f32 else C.BF16 * np.abs(y))
            C.close(C.host(t), y + add, slack, "weight gradient")

        check_dw(dw, b.places(dout), hv)
        # the gradient may take the projections' place
        t_gu = C.dev(gu)
        B.cobalt_expert_down_backward(C.dev(dout), b.t_rows, b.t_off, C.dev(b.w_down), t_gu, None,
                                      t_gu, None, ws, act=kind)
        assert torch.equal(t_gu[:b.used].view(torch.int16), dgu[:b.used].view(torch.int16))

        dx, dw = marked(b.n, b.d), marked(b.E, 2 * b.f, b.d)
        B.cobalt_expert_gate_up_backward(dgu, C.dev(b.x), b.t_rows, b.t_off, C.dev(b.w_in), dx, dw,
                                         ws)
        a = C.host(dgu)
        a[b.used:] = 0
        y, size = X.per_expert(a, b.off, X.wide(b.w_in).transpose(0, 2, 1))
        check_rows(dx, *b.scattered(y, C.BF16 * np.abs(y) + 1.01 * C.product_bound(2 * b.f, size)),
                   "dx")
        check_dw(dw, a, b.places(b.x))

        # fp32 gradients, written and added
        base = b.rng.standard_normal((b.E, b.d, b.f)).astype(np.float32)
        dw = torch.full((b.E, b.d, b.f), float("nan"), device="cuda")
        args = (C.dev(dout), b.t_rows, b.t_off, C.dev(b.w_down), C.dev(gu), C.dev(h), None)
        B.cobalt_expert_down_backward(*args, dw, ws, act=kind, flags=B.GRAD_FLOAT)
        check_dw(dw, b.places(dout), hv, f32=True)
        dw = C.dev(base)
        B.cobalt_expert_down_backward(*args, dw, ws, act=kind, flags=B.GRAD_FLOAT | B.GRAD_ADD)
        check_dw(dw, b.places(dout), hv, add=base, f32=True)
        dw = torch.full((b.E, 2 * b.f, b.d), 2.0, device="cuda")
        B.cobalt_expert_gate_up_backward(dgu, C.dev(b.x), b.t_rows, b.t_off, C.dev(b.w_in), None,
                                         dw, ws, flags=B.GRAD_FLOAT | B.GRAD_ADD)
        check_dw(dw, a, b.places(b.x), add=2.0, f32=True)


def test_no_places():
    """M = 0: nothing is written but the weight gradients, which are zero."""
    E, d, f = 3, 40, 24
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    e = lambda n: torch.empty(0, n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    w_in, w_down = marked(E, 2 * f, d), marked(E, d, f)
    B.cobalt_expert_gate_up(e(d), none, off, w_in, e(f), e(2 * f))
    out = marked(4, d)
    B.cobalt_expert_down(e(f), off, w_down, none, out)
    assert (out == marked(4, d)).all()
    ws = B.expert_backward_workspace_for(0, E, d, f)
    dw, dw_in = marked(E, d, f), torch.ones(E, 2 * f, d, device="cuda")
    B.cobalt_expert_down_backward(e(d), none, off, w_down, e(2 * f), e(f), e(2 * f), dw, ws)
    B.cobalt_expert_gate_up_backward(e(2 * f), e(d), none, off, w_in, e(d), dw_in, ws,
                                     flags=B.GRAD_FLOAT)
    assert not dw.any() and not dw_in.any()


def test_special_values_stay_in_their_rows():
    """A row with infinities and NaN reaches its own outputs only, and a
    weight row its own column only."""
    b = Block(([40, 70], 0, 136, 72), rows=False)
    b.x[5, 3], b.x[60, 7] = 0x7f80, 0x7fc0
    b.w_in[1, 9, 2] = 0x7fc0
    h, gu, _ = run_forward(b, B.ACT_SILU)
    nan = np.isnan(C.host(gu)) | np.isinf(C.host(gu))
    want = np.zeros((b.M, 2 * b.f), bool)
    want[[5, 60]] = True
    want[40:, 9] = True
    assert np.array_equal(nan, want)
    # a row of another expert does not reach a weight gradient
    gu, hh = C.bf16(b.rng, b.M, 2 * b.f), C.bf16(b.rng, b.M, b.f)
    hh[41] = 0x7fc0
    dw = marked(2, b.d, b.f)
    B.cobalt_expert_down_backward(C.dev(C.bf16(b.rng, b.M, b.d)), None, b.t_off, C.dev(b.w_down),
                                  C.dev(gu), C.dev(hh), None, dw,
                                  B.expert_backward_workspace_for(b.M, 2, b.d, b.f))
    nan = np.isnan(C.host(dw))
    assert not nan[0].any() and nan[1].all()


def test_rows_beyond_32_bit_offsets():
    """Rows, gathered and scattered, over 4 GiB from the buffer's start."""
    d, f, n = 8192, 64, 280000
    counts, x = [3, 2], torch.zeros(280000, 8192, dtype=torch.bfloat16, device="cuda")
    rows = np.array([279999, 5, 262144, 270001, 0], np.int32)
    rng = np.random.default_rng(3)
    vals = C.bf16(rng, 5, d)
    x[torch.from_numpy(rows).long().cuda()] = C.dev(vals)
    w_in, w_down = C.bf16(rng, 2, 2 * f, d, scale=d ** -0.5), C.bf16(rng, 2, d, f, scale=0.1)
    off = C.offsets_of(counts)
    h = marked(5, f)
    B.cobalt_expert_gate_up(x, C.dev(rows), C.dev(off), C.dev(w_in), h)
    _, _, want, slack = C.gate_up(X.wide(vals), off, X.wide(w_in), X.SILU)
    C.close(C.host(h), want, slack, "h")
    x.zero_()
    B.cobalt_expert_down(h, C.dev(off), C.dev(w_down), C.dev(rows), x)
    y, size = X.per_expert(C.host(h), off, X.wide(w_down))
    C.close(C.host(x[torch.from_numpy(rows).long().cuda()]), y,
            C.BF16 * np.abs(y) + 1.01 * C.product_bound(f, size), "out")
    assert int((x != 0).any(1).sum()) == 5


def test_offsets_that_are_no_groups():
    """Offsets out of range or decreasing: no access outside the buffers; the
    results of such calls are not defined."""
    b = Block(([30, 34], 0, 64, 64), rows=False)
    for off in ([-5, 20, 900], [64, 10, 64], [2**31 - 1, -2**31, 7]):
        run = C.dev(np.array(off, np.int32))
        guard = marked(b.M + 64, b.f)
        B.cobalt_expert_gate_up(C.dev(b.x), None, run, C.dev(b.w_in), guard[:b.M])
        assert (guard[b.M:] == guard[-1, -1]).all()


def test_repeated_calls_agree_on_any_stream():
    """The same bits again, on a stream of its own, and from a graph that is
    replayed between other work."""
    b = Block(([200, 0, 77, 130], 0, 264, 136))
    T, K = 64, 4
    topk = C.dev(b.rng.integers(0, b.E, (T, K)).astype(np.int32))
    gws = B.expert_group_workspace_for(T, K, b.E)
    rows, tokens = torch.empty(2, T * K, dtype=torch.int32, device="cuda")
    off = torch.empty(b.E + 1, dtype=torch.int32, device="cuda")
    x, w_in, w_down = C.dev(C.bf16(b.rng, T, b.d)), C.dev(b.w_in), C.dev(b.w_down)
    h, gu, out = marked(T * K, b.f), marked(T * K, 2 * b.f), marked(T * K, b.d)
    dgu, dw, dwi = marked(T * K, 2 * b.f), marked(b.E, b.d, b.f), marked(b.E, 2 * b.f, b.d)
    ws = B.expert_backward_workspace_for(T * K, b.E, b.d, b.f)

    def step():
        B.cobalt_expert_group(topk, None, b.E, rows, off, gws, tokens=tokens)
        B.cobalt_expert_gate_up(x, tokens, off, w_in, h, gu)
        B.cobalt_expert_down(h, off, w_down, rows, out)
        B.cobalt_expert_down_backward(out, rows, off, w_down, gu, h, dgu, dw, ws)
        B.cobalt_expert_gate_up_backward(dgu, x, tokens, off, w_in, None, dwi, ws)

    results = (rows, tokens, off, h, gu, out, dgu, dw, dwi)

    def taken():
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        for t in results:
            t.fill_(3)
        return got

    step()
    first = taken()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    second = taken()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    replays = []
    for _ in range(3):
        graph.replay()
        replays.append(taken())
        (torch.randn(256, 256, device="cuda") @ torch.randn(256, 256, device="cuda")).sum().item()
    for got in [second] + replays:
        for a, c in zip(first, got):
            assert torch.equal(a.view(torch.int16), c.view(torch.int16))
