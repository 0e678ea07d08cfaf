"""The experts' operators, as a program around the routing step runs them:
the cases, their inputs, the operators written out in elementary torch
operations, and the same results in 64 bits.

Five kinds of pass:

  forward   rows grouped by expert, gate and up projections with activation
            and product (h), down projection (out). `serve` gathers token
            rows and writes one row per pair; otherwise the packed rows of
            the dispatch go in and out and the projections are kept for the
            backward pass
  backward  gradients of the projections, of both weights and of the rows
  quantize  bf16 rows to microscaled 4-bit rows and back
  mx        the forward pass on microscaled 4-bit rows and weights
  combine   the gradients of the combine: of the expert rows and of the gates

A stored bf16 or 4-bit result is what the next operator of a pass reads, here
as in the library.
"""
import math

import torch

own = False

BLOCK = 32                                  # values that share a scale
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(op, T, K, E, d, f, *, alpha=0.3, drop=0.0, serve=False, act="silu", **name):
    return dict(name, op=op, T=T, K=K, E=E, d=d, f=f, alpha=alpha, drop=drop, serve=serve,
                act=act)


def listed():
    return [
        # one new token of a serving program: the weights of K experts are read
        _case("forward", 1, 8, 64, 4096, 1024, serve=True, name="forward-1-e64"),
        # an odd batch of a serving program, uneven experts, widths that fill
        # no tile, and pairs that a capacity limit dropped
        _case("forward", 1021, 6, 64, 2048, 1000, alpha=0.6, drop=0.02, serve=True, act="gelu",
              name="forward-1021-e64-odd"),
        # one rank of the widest workload: its share of a step's rows
        _case("forward", 8192, 2, 8, 7168, 2048, name="forward-8192-e8"),
        # the benchmark's smallest width, an odd number of tokens
        _case("backward", 509, 2, 16, 512, 256, name="backward-509-e16"),
        # the middle workload's experts in a training step
        _case("backward", 4096, 6, 64, 2048, 1024, name="backward-4096-e64"),
        # the backward pass of the widest workload's rank
        _case("backward", 8192, 2, 8, 7168, 2048, name="backward-8192-e8"),
        # the rows of a small decoding batch
        _case("quantize", 33, 1, 1, 4096, 1024, name="quantize-33"),
        # the rows of a long prompt, before they are dispatched
        _case("quantize", 65536, 1, 1, 7168, 2048, name="quantize-65536"),
        # one new token on 4-bit experts
        _case("mx", 1, 8, 128, 4096, 1024, serve=True, name="mx-1-e128"),
        # a prompt on 4-bit experts
        _case("mx", 8192, 2, 8, 7168, 2048, serve=True, name="mx-8192-e8"),
        # an uneven batch, dropped pairs
        _case("combine", 1021, 6, 64, 1032, 8, drop=0.02, name="combine-1021-k6"),
        # an eighth of the headline workload's step
        _case("combine", 16384, 8, 256, 7168, 8, name="combine-16384-k8"),
    ]


def _log_int(rng, lo, hi, unit=1):
    """A multiple of unit in [lo, hi], evenly over its logarithm; never 3072,
    a width that no workload here has."""
    while True:
        n = unit * max(1, int(round(lo * (hi / lo) ** rng.random() / unit)))
        if n != 3072:
            return n


# the products and the row values of the largest listed case, which no drawn one passes
_MOST_MACS = 16384 * 7168 * 2048
_MOST_WEIGHTS = 128 * 4096 * 1024
_MOST_ROWS = 65536 * 7168


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "mx", "mx", "quantize",
                     "combine"])
    unit = 32 if op in ("mx", "quantize") else 8
    d = _log_int(rng, 256, 7168, unit)
    f = _log_int(rng, 128, 2048, unit)
    if op == "quantize":
        return _case(op, min(_log_int(rng, 1, 65536), _MOST_ROWS // d), 1, 1, d, 1024)
    E = rng.choice([4, 8, 16, 48, 64, 128, 256])
    while E * d * f > _MOST_WEIGHTS:
        E //= 2
    E = max(E, 4)
    K = rng.choice([1, 2, 3, 4])
    serve = op == "mx" or (op == "forward" and rng.random() < 0.5)
    T = _log_int(rng, 1 if serve else 64, 16384)
    drop = rng.choice([0.0, 0.0, 0.01])
    if op == "combine":
        K = rng.choice([1, 2, 4, 6, 7, 8])
        return _case(op, min(T, _MOST_ROWS // (K * d)), K, 64, d, 8, drop=drop)
    T = max(1, min(T, _MOST_MACS // (K * d * f)))
    return _case(op, T, K, E, d, f, alpha=rng.choice([0.0, 0.3, 0.6]), drop=drop, serve=serve,
                 act=rng.choice(["silu", "silu", "gelu"]))


# ------------------------------------------------------------------- inputs
def _routing(case, gen):
    """Each token's K distinct experts, popular ones more often; -1 where a
    pair was dropped."""
    T, K, E = case["T"], case["K"], case["E"]
    order = torch.randperm(E, generator=gen, device="cuda").float()
    logits = torch.randn(T, E, generator=gen, device="cuda") - case["alpha"] * torch.log1p(order)
    topk = torch.topk(logits, K, dim=1).indices.to(torch.int32)
    if case["drop"]:
        gone = torch.rand(T, K, generator=gen, device="cuda") < case["drop"]
        topk = torch.where(gone, torch.full_like(topk, -1), topk)
    return topk.contiguous()


def _normal(gen, *shape, scale=1.0):
    t = torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
    for part in t.split(max(1, (1 << 28) // max(1, t[0].numel()))):  # fp32 draws, a piece at a time
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * scale)
    return t


def _hidden(gen, n, d):
    """Hidden states: normal values, and one channel in 64 sixteen times as large."""
    x = _normal(gen, n, d)
    x[:, 5::64] *= 16
    return x


def _zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    T, K, E, d, f, op = (case[k] for k in ("T", "K", "E", "d", "f", "op"))
    M = T * K
    st = dict(case, M=M)
    if op == "quantize":
        st.update(x=_hidden(gen, T, d), q=_zeros(T, d // 2, dtype=torch.uint8),
                  s=_zeros(T, d // BLOCK, dtype=torch.uint8), back=_zeros(T, d))
        return st
    st["topk"] = _routing(case, gen)
    perm = torch.randperm(M, generator=gen, device="cuda").to(torch.int32).view(T, K)
    if op == "combine":
        st.update(pos=torch.where(st["topk"] < 0, torch.full_like(perm, -1), perm),
                  gates=torch.softmax(torch.randn(T, K, generator=gen, device="cuda"), 1),
                  dy=_normal(gen, T, d, scale=1 / 64), eo=_normal(gen, M, d),
                  deo=_zeros(M, d), dgates=_zeros(T, K, dtype=torch.float32))
        return st
    # the most rows of an expert: a program knows its capacity
    st["cap"] = max(1, int(torch.bincount(st["topk"].flatten().long() + 1,
                                          minlength=E + 1)[1:].max()))
    st.update(rows=_zeros(M, dtype=torch.int32), tokens=_zeros(M, dtype=torch.int32),
              offsets=_zeros(E + 1, dtype=torch.int32), pos=None if case["serve"] else perm)
    w_in = _normal(gen, E, 2 * f, d, scale=1 / math.sqrt(d))
    w_down = _normal(gen, E, d, f, scale=1 / math.sqrt(f))
    if op == "mx":
        # weights laid out once, when the model is loaded
        st["w_in"], st["w_in_scale"] = _quantize(w_in)
        st["w_down"], st["w_down_scale"] = _quantize(w_down)
        st.update(x=_hidden(gen, T, d), h=_zeros(M, f), out=_zeros(M, d),
                  xq=_zeros(T, d // 2, dtype=torch.uint8),
                  xs=_zeros(T, d // BLOCK, dtype=torch.uint8),
                  hq=_zeros(M, f // 2, dtype=torch.uint8),
                  hs=_zeros(M, f // BLOCK, dtype=torch.uint8))
        return st
    st.update(w_in=w_in, w_down=w_down)
    if op == "forward":
        st.update(x=_normal(gen, T if case["serve"] else M, d), h=_zeros(M, f), out=_zeros(M, d),
                  gate_up=None if case["serve"] else _zeros(M, 2 * f))
        return st
    # backward: what the forward pass kept, and the gradient of its output
    rows, _, offsets, _ = _group(st["topk"], perm, E)
    st.update(rows=rows, offsets=offsets, x=_normal(gen, M, d), gate_up=_normal(gen, M, 2 * f),
              dout=_normal(gen, M, d, scale=1 / 64))
    g, u = st["gate_up"].float().split(f, dim=1)
    st["h"] = (_act(g, case["act"]) * u).to(torch.bfloat16)
    st.update(dgate_up=_zeros(M, 2 * f), dx=_zeros(M, d), dw_in=_zeros(E, 2 * f, d),
              dw_down=_zeros(E, d, f))
    return st


# -------------------------------------------------------------- plain forms
def _act(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g)))


def _act_slope(g, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _group(topk, pos, E):
    """rows and tokens of the pairs in order of (expert, pair), -1 behind the
    last kept pair; offsets of the experts; expert of each place (E: none)."""
    T, K = topk.shape
    e = topk.flatten().long()
    e = torch.where((e < 0) | (e >= E), torch.full_like(e, E), e)
    e, p = torch.sort(e, stable=True)
    count = torch.zeros(E + 1, dtype=torch.int64, device=e.device)
    count.scatter_add_(0, e, torch.ones_like(e))
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=e.device)
    offsets[1:] = torch.cumsum(count[:E], 0)
    at = p if pos is None else pos.flatten()[p].long()
    none = torch.full_like(p, -1)
    rows = torch.where(e < E, at, none).to(torch.int32)
    tokens = torch.where(e < E, p // K, none).to(torch.int32)
    return rows, tokens, offsets.to(torch.int32), e


def _places(e, offsets, E, cap):
    """Where each sorted pair lies in [E][cap] rows (the row behind them for a
    dropped pair)."""
    i = torch.arange(e.numel(), device=e.device)
    start = torch.cat([offsets[:E].long(), torch.zeros(1, dtype=torch.int64, device=e.device)])
    return torch.where(e < E, e * cap + i - start[e], torch.full_like(e, E * cap))


def _padded(a, at, E, cap):
    out = torch.zeros(E * cap + 1, a.shape[1], dtype=torch.float32, device=a.device)
    out[at] = a
    return out[:-1].view(E, cap, a.shape[1])


def _taken(a, at):
    """The rows `at` of [E][cap] padded ones, zero for dropped pairs."""
    E, cap, n = a.shape
    a = torch.cat([a.reshape(E * cap, n), torch.zeros(1, n, dtype=a.dtype, device=a.device)])
    return a[at]


def _product(a, w, e, at, cap, turn=True):
    """a[i] times the weights of its expert. w: [E][n][k] weights, or 4-bit
    ones with their scales, for [M][k] rows; with turn=False [E][k][n]."""
    w = w if isinstance(w, tuple) else (w,)
    E = w[0].shape[0]
    few = a.shape[0] <= E  # few rows: only their experts' weights
    if few:
        w = tuple(t[e.clamp(max=E - 1)] for t in w)
    w = _dequantize(*w) if len(w) == 2 else w[0].float()
    w = w.transpose(1, 2) if turn else w
    if few:
        y = torch.bmm(a[:, None, :], w)[:, 0]
        return torch.where((e < E)[:, None], y, torch.zeros_like(y))
    return _taken(torch.bmm(_padded(a, at, E, cap), w), at)


def _gathered(x, idx):
    return torch.where((idx >= 0)[:, None], x[idx.long().clamp(min=0)].float(),
                       torch.zeros((), device=x.device))


def _scattered(rows, y, n):
    """y[i] to row rows[i]; rows without a pair stay zero."""
    out = torch.zeros(n + 1, y.shape[1], dtype=y.dtype, device=y.device)
    out[torch.where(rows < 0, torch.full_like(rows, n), rows).long()] = y
    return out[:n]


def _quantize(x):
    """Blocks of 32 values: the scale is 2^(floor(log2(largest)) - 2), each
    value the nearest of E2M1 (ties to the even code). Codes two to a byte,
    scales as biased exponents, 255 for a block with an infinity or NaN."""
    v = x.float().reshape(*x.shape[:-1], -1, BLOCK)
    big = v.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(v).all(-1, keepdim=True)
    big = torch.where(fine, big, torch.ones_like(big))
    ex = (torch.frexp(big).exponent - 3).clamp(-127, 127)
    ex = torch.where(big > 0, ex, torch.full_like(ex, -127))
    m = torch.where(fine, torch.ldexp(v.abs(), -ex), torch.zeros_like(v))
    code = (m > 0.25).to(torch.uint8)
    for level, even in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True),
                        (5.0, False)):
        code += (m >= level) if even else (m > level)
    code += 8 * (torch.signbit(v) & fine).to(torch.uint8)
    code = code.reshape(*x.shape[:-1], -1)
    scale = torch.where(fine, ex + 127, torch.full_like(ex, 255)).to(torch.uint8)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), scale.squeeze(-1).contiguous()


def _dequantize(q, s):
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float32, device=q.device)
    code = torch.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], -1, BLOCK).long()
    scale = torch.ldexp(torch.ones((), device=q.device), s.int() - 127)
    scale = torch.where(s == 255, torch.full_like(scale, math.nan), scale)
    return (lut[code] * scale[..., None]).reshape(*q.shape[:-1], -1)


def _plain(st):
    op, act = st["op"], st["act"]
    bf16 = torch.bfloat16
    if op == "quantize":
        return {"values": _dequantize(*_quantize(st["x"])).to(bf16)}
    if op == "combine":
        T, K, pos = st["T"], st["K"], st["pos"].flatten()
        dy = st["dy"].float().repeat_interleave(K, 0)
        dgates = (dy * _gathered(st["eo"], pos)).sum(1).view(T, K)
        deo = _scattered(pos, st["gates"].reshape(-1, 1) * dy, st["M"])
        return {"deo": deo.to(bf16), "dgates": dgates}
    E, M, f, cap = st["E"], st["M"], st["f"], st["cap"]
    if op == "backward":
        rows, offsets = st["rows"], st["offsets"]
        e = torch.searchsorted(offsets[1:].contiguous(), torch.arange(M, device="cuda",
                                                                      dtype=torch.int32),
                               right=True)
        at = _places(e, offsets, E, cap)
        dout = _gathered(st["dout"], rows)
        g, u = st["gate_up"].float().split(f, dim=1)
        dh = _product(dout, st["w_down"], e, at, cap, turn=False)
        dgu = torch.cat([dh * u * _act_slope(g, act), dh * _act(g, act)], 1).to(bf16)
        x = _padded(_gathered(st["x"], rows), at, E, cap)
        dw_down = torch.bmm(_padded(dout, at, E, cap).transpose(1, 2),
                            _padded(st["h"].float(), at, E, cap))
        dw_in = torch.bmm(_padded(dgu.float(), at, E, cap).transpose(1, 2), x)
        dx = _scattered(rows, _product(dgu.float(), st["w_in"], e, at, cap, turn=False), M)
        return {"dgate_up": dgu, "dw_down": dw_down.to(bf16), "dx": dx.to(bf16),
                "dw_in": dw_in.to(bf16)}
    rows, tokens, offsets, e = _group(st["topk"], st["pos"], E)
    at = _places(e, offsets, E, cap)
    idx = tokens if st["serve"] else rows
    w_in, w_down = st["w_in"], st["w_down"]
    if op == "mx":
        w_in, w_down = (w_in, st["w_in_scale"]), (w_down, st["w_down_scale"])
        a = _gathered(_dequantize(*_quantize(st["x"])), idx)
    else:
        a = _gathered(st["x"], idx)
    gu = _product(a, w_in, e, at, cap)
    h = (_act(gu[:, :f], act) * gu[:, f:]).to(bf16)
    a = _dequantize(*_quantize(h)) if op == "mx" else h.float()
    out = _scattered(rows, _product(a, w_down, e, at, cap), M)
    got = {"rows": rows, "offsets": offsets, "h": h, "out": out.to(bf16)}
    return got if st["serve"] else dict(got, gate_up=gu.to(bf16))


# ---------------------------------------------------------- the library's calls
def _library(st):
    from paper_2609_36959_amd import binding as B
    op = st["op"]
    if op == "quantize":
        B.cobalt_mx_quantize(st["x"], st["q"], st["s"])
        B.cobalt_mx_dequantize(st["q"], st["s"], st["back"])
        return {"values": st["back"]}
    if op == "combine":
        B.cobalt_combine_backward(st["dy"], st["eo"], st["pos"], st["gates"], st["deo"],
                                  st["dgates"])
        return {"deo": st["deo"], "dgates": st["dgates"]}
    act = B.ACT_SILU if st["act"] == "silu" else B.ACT_GELU
    rows, offsets = st["rows"], st["offsets"]
    if op == "backward":
        if "ws" not in st:
            st["ws"] = B.expert_backward_workspace_for(st["M"], st["E"], st["d"], st["f"])
        B.cobalt_expert_down_backward(st["dout"], rows, offsets, st["w_down"], st["gate_up"],
                                      st["h"], st["dgate_up"], st["dw_down"], st["ws"], act=act)
        B.cobalt_expert_gate_up_backward(st["dgate_up"], st["x"], rows, offsets, st["w_in"],
                                         st["dx"], st["dw_in"], st["ws"])
        return {k: st[k] for k in ("dgate_up", "dw_down", "dx", "dw_in")}
    if "ws" not in st:
        st["ws"] = B.expert_group_workspace_for(st["T"], st["K"], st["E"])
    B.cobalt_expert_group(st["topk"], st["pos"], st["E"], rows, offsets, st["ws"],
                          tokens=st["tokens"])
    idx = st["tokens"] if st["serve"] else rows
    if op == "mx":
        B.cobalt_mx_quantize(st["x"], st["xq"], st["xs"])
        B.cobalt_mx_gate_up(st["xq"], st["xs"], idx, offsets, st["w_in"], st["w_in_scale"],
                            st["h"], act=act)
        B.cobalt_mx_quantize(st["h"], st["hq"], st["hs"])
        B.cobalt_mx_down(st["hq"], st["hs"], offsets, st["w_down"], st["w_down_scale"], rows,
                         st["out"])
    else:
        B.cobalt_expert_gate_up(st["x"], idx, offsets, st["w_in"], st["h"], st["gate_up"], act=act)
        B.cobalt_expert_down(st["h"], offsets, st["w_down"], rows, st["out"])
    got = {"rows": rows, "offsets": offsets, "h": st["h"], "out": st["out"]}
    return got if st["serve"] else dict(got, gate_up=st["gate_up"])


def run(st):
    return _library(st) if own else _plain(st)


# -------------------------------------------------------------------- work
def work(case):
    T, K, E, d, f, op = (case[k] for k in ("T", "K", "E", "d", "f", "op"))
    M = T * K
    if op == "quantize":  # in, codes and scales out and in again, values out
        return {"bytes": T * d * (2 + 2 * (0.5 + 1 / BLOCK) + 2), "flops": 2 * T * d}
    if op == "combine":
        return {"bytes": 2 * T * d + 2 * 2 * M * d + 3 * 4 * M, "flops": 3 * M * d}
    touched = E * (1 - (1 - K / E) ** T)  # experts with a row, were they equally likely
    if op == "backward":
        data = 2 * M * (2 * d + 2 * f + 2 * f + f + d) + 2 * 3 * d * f * (touched + E)
        return {"bytes": data + 4 * M, "flops": 12 * M * d * f}
    index = 4 * M * (3 if not case["serve"] else 2)
    if op == "mx":  # rows in, out and 4-bit copies of x and h
        size = 0.5 + 1 / BLOCK
        data = T * d * (2 + 2 * size) + M * f * (2 + 2 + 2 * size) + 2 * M * d
        return {"bytes": data + size * 3 * d * f * touched + index, "flops": 6 * M * d * f}
    data = 2 * ((T if case["serve"] else M) * d + 2 * M * f + M * d)
    data += 0 if case["serve"] else 2 * M * 2 * f
    return {"bytes": data + 2 * 3 * d * f * touched + index, "flops": 6 * M * d * f}


# ----------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The results from the definitions, expert by expert in 64 bits."""
    st = prepare(case, seed)
    op, T, K, E, M, d, f = (st[k] for k in ("op", "T", "K", "E", "M", "d", "f"))
    f64 = torch.float64

    def nearest(v):  # 4-bit values that v stands for, from the definition
        v = v.to(f64).reshape(v.shape[0], -1, BLOCK)
        big = v.abs().amax(-1, keepdim=True)
        ex = torch.floor(torch.log2(torch.where(big > 0, big, torch.ones_like(big)))) - 2
        ex = torch.where(big > 0, ex, torch.full_like(ex, -127)).clamp(-127, 127)
        ratio = v / torch.pow(torch.full_like(ex, 2), ex)
        size = ratio.abs()
        step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
        # round() takes ties to even multiples of the step, which are even codes
        size = (torch.round(size / step) * step).clamp(max=6)
        return (torch.sign(ratio) * size * torch.pow(torch.full_like(ex, 2), ex)).flatten(1)

    def activation(g):
        if case["act"] == "silu":
            return g * torch.sigmoid(g)
        return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))

    if op == "quantize":
        return {"values": torch.cat([nearest(p) for p in st["x"].split(8192)])}
    if op == "combine":
        deo, dgates = torch.zeros(M, d, dtype=f64, device="cuda"), torch.zeros(T, K, dtype=f64,
                                                                               device="cuda")
        for j in range(K):
            t = torch.nonzero(st["pos"][:, j] >= 0)[:, 0]
            at = st["pos"][t, j].long()
            dy = st["dy"][t].to(f64)
            deo[at] = dy * st["gates"][t, j:j + 1].to(f64)
            dgates[t, j] = (dy * st["eo"][at].to(f64)).sum(1)
        return {"deo": deo, "dgates": dgates}
    flat = st["topk"].flatten()

    if op == "backward":
        r = {"dgate_up": torch.zeros(M, 2 * f, dtype=f64, device="cuda"),
             "dw_down": torch.zeros(E, d, f, dtype=f64, device="cuda"),
             "dx": torch.zeros(M, d, dtype=f64, device="cuda"),
             "dw_in": torch.zeros(E, 2 * f, d, dtype=f64, device="cuda")}
        lo = 0
        for e in range(E):
            hi = lo + int((flat == e).sum())
            at = st["rows"][lo:hi].long()
            dout, x = st["dout"][at].to(f64), st["x"][at].to(f64)
            with torch.enable_grad():
                gu = st["gate_up"][lo:hi].to(f64).requires_grad_()
                h = activation(gu[:, :f]) * gu[:, f:]
                dgu, = torch.autograd.grad(h, gu, dout @ st["w_down"][e].to(f64))
            r["dgate_up"][lo:hi] = dgu
            dgu = dgu.to(torch.bfloat16).to(f64)  # as stored
            r["dw_down"][e] = dout.t() @ st["h"][lo:hi].to(f64)
            r["dx"][at] = dgu @ st["w_in"][e].to(f64)
            r["dw_in"][e] = dgu.t() @ x
            lo = hi
        return r

    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=f64, device="cuda")

    def weights(name, e):
        w = st[name][e]
        if op != "mx":
            return w.to(f64)
        w = torch.stack([lut[(w & 15).long()], lut[(w >> 4).long()]], -1).flatten(1)
        s = torch.pow(torch.tensor(2.0, dtype=f64, device="cuda"),
                      st[name + "_scale"][e].to(f64) - 127)
        return w * s.repeat_interleave(BLOCK, 1)

    r = {"rows": None, "offsets": None, "h": torch.zeros(M, f, dtype=f64, device="cuda"),
         "out": torch.zeros(M, d, dtype=f64, device="cuda")}
    if not st["serve"]:
        r["gate_up"] = torch.zeros(M, 2 * f, dtype=f64, device="cuda")
    lo = 0
    for e in range(E):
        p = torch.nonzero(flat == e)[:, 0]
        if not p.numel():
            continue
        hi = lo + p.numel()
        at = p if st["pos"] is None else st["pos"].flatten()[p].long()
        x = st["x"][p // K if st["serve"] else at]
        gu = (nearest(x) if op == "mx" else x.to(f64)) @ weights("w_in", e).t()
        h = activation(gu[:, :f]) * gu[:, f:]
        r["h"][lo:hi] = h
        if not st["serve"]:
            r["gate_up"][lo:hi] = gu
        h = h.to(torch.bfloat16)  # as stored
        r["out"][at] = (nearest(h) if op == "mx" else h.to(f64)) @ weights("w_down", e).t()
        lo = hi
    return r
