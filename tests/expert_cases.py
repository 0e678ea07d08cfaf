"""Inputs and bounds shared by the tests of the experts' operators."""
import numpy as np
import torch

import oracle.experts as X

# How far a bf16 result may be from the exact one: half a unit in the last
# place, at most 2^-8 of it, on top of the fp32 error of what is rounded. A
# product of n terms accumulated in fp32 in any order is off by at most
# n * 2^-23 of the sum of the terms' magnitudes (each addition by 2^-24 of a
# partial sum, which never exceeds that sum; twice that for the matrix cores,
# whose adds may truncate). The activations' exponential, reciprocal and
# products are eight fp32 operations of at most 2^-22 each, the exponential's
# argument adding |z| * 2^-23 with |z| under 90: 2^-15 of the value covers
# both. Values of 2^-120 and below may flush.
BF16 = 2.0 ** -8
ACT = 2.0 ** -15
TINY = 2.0 ** -120


def product_bound(terms, size):
    return terms * 2.0 ** -23 * size


def offsets_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def bf16(rng, *shape, scale=1.0):
    """Random normal bf16 values, as bits."""
    v = (rng.standard_normal(shape) * scale).astype(np.float32)
    return torch.from_numpy(v).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def dev(bits):
    """A device tensor of bf16 bits, or of any other array."""
    if bits is None:
        return None
    if bits.dtype == np.uint16:
        return torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).cuda()
    return torch.from_numpy(np.ascontiguousarray(bits)).cuda()


def host(t):
    """Values of a device tensor, bf16 and fp32 ones as float64."""
    t = t.detach().cpu()
    if t.dtype == torch.bfloat16:
        return X.wide(t.view(torch.int16).numpy().view(np.uint16))
    return t.numpy().astype(np.float64) if t.dtype == torch.float32 else t.numpy()


def close(got, want, slack, what):
    """|got - want| within `slack` on every element, no NaN unless wanted."""
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places"
    off = np.abs(got - want)
    over = np.where(nan, False, ~(off <= slack + TINY))
    if over.any():
        i = tuple(np.argwhere(over)[0])
        raise AssertionError(f"{what}: {over.sum()} of {over.size} outside, first at {i}: "
                             f"{got[i]} for {want[i]}, bound {np.broadcast_to(slack, got.shape)[i]}")


def gate_up(a, offsets, w_in, kind):
    """g, u and h of the places' rows a, with the bounds of their bf16 forms."""
    f, d = w_in.shape[1] // 2, w_in.shape[2]
    gu, size = X.per_expert(a, offsets, w_in)
    err = product_bound(d, size)
    g, u = gu[:, :f], gu[:, f:]
    ag = X.act(g, kind)
    h = ag * u
    # |a'| is at most 1.13
    h_err = 1.13 * err[:, :f] * (np.abs(u) + err[:, f:]) + np.abs(ag) * err[:, f:] \
        + ACT * np.abs(h)
    return gu, BF16 * np.abs(gu) + 1.01 * err, h, BF16 * np.abs(h) + 1.01 * h_err


def down_gradient(dout, offsets, w_down, gate_up, kind):
    """dgate_up of the places' gradients dout, with its bound."""
    f = w_down.shape[2]
    dh, size = X.per_expert(dout, offsets, w_down.transpose(0, 2, 1))
    err = product_bound(w_down.shape[1], size)
    g, u = gate_up[:, :f], gate_up[:, f:]
    slope, ag = X.act_slope(g, kind), X.act(g, kind)
    want = np.concatenate([dh * u * slope, dh * ag], 1)
    # the slope is a sum of terms of size up to 1 + |g| that may cancel
    e_slope = ACT * (1 + np.abs(g))
    bound = np.concatenate([np.abs(u) * (err * (np.abs(slope) + e_slope) + np.abs(dh) * e_slope),
                            np.abs(ag) * err + np.abs(dh * ag) * ACT], 1)
    return want, BF16 * np.abs(want) + 1.01 * bound
