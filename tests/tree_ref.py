"""Plain 64-bit forms of the operators that check drafted tokens, on the CPU, with bounds of what fp32 sums and bf16 operands
may differ by. A bf16 rounding is off by at most 2^-8 of the value, an fp32 one by 2^-24; a tensor-core instruction that adds
16 products to an accumulator is allowed 17 roundings of the largest sum of magnitudes."""
import math

import torch

BF16, FP32 = 2.0 ** -8, 2.0 ** -24


# ---------------------------------------------------------------------------------------------- 4-bit weights
def w4_values(codes, scales, zeros, group):
    """fp64 weights of plain codes [N, K], scales [N, groups], zeros [N, groups] or None."""
    at = torch.arange(codes.shape[1]) // group
    z = 8.0 if zeros is None else zeros.double()[:, at]
    return (codes.double() - z) * scales.double()[:, at]


def act(g, kind):
    if kind == 0:
        return g * torch.sigmoid(g)
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def gemv(x, w, group):
    """(y, bound) of x [B, K] w [N, K]^T: per element 17 roundings for each 16 inputs of a group, one for each group that joins
    the sum and some for the slices, of the sum of magnitudes."""
    x = x.double()
    y, mag = x @ w.t(), x.abs() @ w.abs().t()
    return y, (17 * group / 16 + -(-x.shape[1] // group) + 16) * FP32 * mag


def gated(y, e, kind):
    """(out, bound) of the gated form of y [B, N] with errors e: blocks of 128 gate and 128 up columns. Both activations have a
    slope of at most 1.13; their fp32 forms are allowed 16 roundings."""
    y, e = (v.view(v.shape[0], -1, 2, 128) for v in (y, e))
    g, u, eg, eu = y[:, :, 0], y[:, :, 1], e[:, :, 0], e[:, :, 1]
    a = act(g, kind)
    out = a * u
    err = 1.13 * eg * (u.abs() + eu) + (a.abs() + 16 * FP32 * g.abs()) * eu + 16 * FP32 * (a.abs() + g.abs()) * u.abs()
    return out.flatten(1), (err + BF16 * (out.abs() + err)).flatten(1) + 1e-38


# ---------------------------------------------------------------------------------------------- rows of a tree
def random_tree(rows, g):
    return [int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(rows)]


def sees(parents):
    """bool [rows, rows] and depths of a tree, by walking up from each row."""
    n = len(parents)
    m, depth = torch.zeros(n, n, dtype=torch.bool), []
    for i in range(n):
        k, d = i, -1
        while k >= 0:
            m[i, k] = True
            k, d = parents[k], d + 1
        depth.append(d)
    return m, torch.tensor(depth, dtype=torch.int32)


def pack_bits(m, words):
    """int32 [rows, words] of bool [rows, <= 32 words]."""
    m = torch.nn.functional.pad(m, (0, words * 32 - m.shape[1])).view(m.shape[0], words, 32).long()
    v = (m << torch.arange(32)).sum(-1)
    return torch.where(v >= 2 ** 31, v - 2 ** 32, v).to(torch.int32)


def turned(x, cs, gain, eps):
    """(rotated rows, bound of their fp32 form) of x [rows, heads, hd] fp64; cs [rows, hd / 2, 2]."""
    hd = x.shape[-1]
    if gain is not None:
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps) * gain.double()
    a, b = x.chunk(2, -1)
    c, s = cs[:, None, :, 0].double(), cs[:, None, :, 1].double()
    rel = (hd + 8) * FP32 if gain is not None else 0.0
    mag = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1), (rel + 4 * FP32) * mag


def attend(q, k, v, seen):
    """(out, bound) of rows q [R, hd] over k, v [n, hd] of one head. Scores are fp32 sums of exact products, weights bf16."""
    hd = q.shape[-1]
    q, k, v = q.double(), k.double(), v.double()
    s = q @ k.t() / math.sqrt(hd)
    mag = (q.abs() @ k.abs().t() / math.sqrt(hd)).masked_fill(~seen, 0)
    delta = (17 * hd / 16 + 8) * FP32 * mag.amax(-1, keepdim=True)                     # error of an exponent
    p = torch.nan_to_num(torch.softmax(s.masked_fill(~seen, -math.inf), -1))
    out, pv = p @ v, p @ v.abs()
    n = k.shape[0]
    rel = 2 * torch.expm1(2 * delta) + (17 * n / 16 + 64) * FP32 + BF16
    return out, rel * (pv + out.abs()) + BF16 * out.abs() + 1e-30
