"""The 8-bit paged cache in plain 64-bit arithmetic on the CPU, sequence by sequence, from its definition: the reference of
tests/test_gpu_cache8.py. Rounding to E4M3 is the format's (3 fraction bits, exponents >= -6, ties to even, saturating)."""
import math

import torch

BLOCK = 16
F32 = 2.0 ** -24             # half a step of fp32, relative
DECODE_SHIFT = 14            # the single-query kernel's weights are stored times 2^14, the prompt kernel's times 2^7


def round_e4m3(y):
    _, e = torch.frexp(y)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def scale_exp(amax):
    """E8M0 byte of the smallest power of two s >= 2^-64 with amax <= 448 s (2^120 for an infinity)."""
    if amax == 0:
        return 63
    if math.isinf(amax):
        return 247
    k = -64
    if amax > 448 * 2.0 ** -64:
        k = math.ceil(math.log2(amax / 448))
        while amax > 448 * 2.0 ** k:
            k += 1
        while k > -64 and amax <= 448 * 2.0 ** (k - 1):
            k -= 1
    return 127 + k


def code_values(u8):
    """Values of E4M3 codes."""
    u = u8.long()
    e, m = (u >> 3) & 15, (u & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e.double() - 10))
    v = torch.where((u & 127) == 127, torch.full_like(v, math.nan), v)
    return torch.where(u >= 128, -v, v)


def read(codes, scales, table_row, n):
    """fp64 values [n, n_kv, hd] of positions 0 .. n-1; codes [pages, n_kv, page, hd] of one layer."""
    page = codes.shape[2]
    pos = torch.arange(n)
    pg, slot = table_row.long()[pos // page], pos % page
    return code_values(codes[pg, :, slot]) * torch.exp2(scales[pg, :, slot // BLOCK].double() - 127)[..., None]


def rotate(x, gain, eps, cs):
    """Per-head RMSNorm (gain or None) and rotation of x [heads, hd] by cs [hd/2, 2], fp64."""
    if gain is not None:
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps) * gain.double()
    h = x.shape[-1] // 2
    z = torch.complex(x[:, :h].contiguous(), x[:, h:].contiguous()) * torch.complex(cs[:, 0].double(), cs[:, 1].double())
    return torch.cat([z.real, z.imag], -1)


def rotate_error(x, gain, eps, cs):
    """Bound of what fp32 arithmetic of `rotate` can be off, elementwise: the mean square is a sum of hd squares ((hd + 2)
    half steps relative, halved by the root), rsqrt and its argument 4, three products 3; the rotation two products and a
    sum of values of size |a| + |b|: 3. The table is an input."""
    if gain is not None:
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps) * gain.double()
    hd = x.shape[-1]
    a, b = x[:, :hd // 2].abs(), x[:, hd // 2:].abs()
    n = (hd + 2) / 2 + 7 + 3 if gain is not None else 3
    c, s = cs[:, 0].double().abs(), cs[:, 1].double().abs()
    return n * F32 * torch.cat([a * c + b * s, b * c + a * s], -1) + 1e-37


def read_exponents(scales, table_row, page, n):
    """Exponents of the scales [n, n_kv] of positions 0 .. n-1."""
    pos = torch.arange(n)
    return scales[table_row.long()[pos // page], :, pos % page // BLOCK].double() - 127


def attend(q, k, v, seen, ev, shift):
    """q [heads, hd], k and v [n, heads, hd] (one kv head per query head), seen [n] -> (out, bound) [heads, hd].
    ev [n, heads]: exponents of V's scales. shift: the largest weight is stored as 2^shift at least.

    bound: the weights are rounded to f16 (2^-11 relative), the scores are fp32 sums of hd products times two factors
    ((hd + 4) half steps of sum |q||k| / sqrt(hd), an absolute error of the exponent, so a relative one of the weight, of
    the numerator and of the denominator), exp2 is good to 2^-21, sums of n weights and values of them are fp32
    (their tree and tile order: 64 half steps are more than any path has: 16 MMA steps of K = 16 per 256 keys, accumulated,
    cost less than n / 16 of them, so n / 16 + 64), the result is rounded to bf16 (2^-8).

    Weights below f16's smallest normal value are off by up to 2^-25 absolutely. What is stored for key j is
    w_j = A p_j 2^ev_j, A such that the largest is 2^shift or more: A >= 2^shift / max_j p_j 2^ev_j. The result is
    sum_j w_j c_j / A with c_j the codes' values, so 2^-25 in every w_j costs at most 2^-25 sum_j |c_j| / A
    <= 2^(-25 - shift) max_j (p_j 2^ev_j) sum_j |c_j|.

    The kernels hold an element of q as the sum of two E4M3 codes after a power-of-two scale that brings the
    head's largest element to 2^7 or more. The first code leaves at most 2^-4 of the element, four bits of a bf16 element's
    eight, which the second holds unless it is below the smallest normal code: then it is off by at most half a step of
    2^-9, 2^-17 of the head's largest. That is an absolute error of the score of 2^-17 max |q| sum |k| / sqrt(hd)."""
    hd = q.shape[-1]
    if not bool(seen.any()):
        return torch.zeros_like(q), torch.zeros_like(q)
    k, v, ev = k[seen], v[seen], ev[seen]
    s = torch.einsum("hd,nhd->nh", q, k) / math.sqrt(hd)
    p = torch.softmax(s, 0)
    out = torch.einsum("nh,nhd->hd", p, v)
    size = torch.einsum("hd,nhd->nh", q.abs(), k.abs()).amax(0) / math.sqrt(hd)              # [heads]
    split = 2.0 ** -17 * q.abs().amax(1) * k.abs().sum(2).amax(0) / math.sqrt(hd)
    rel = 2.0 ** -11 + 2.0 ** -20 + 2 * ((hd + 4) * F32 * size + split) + 2 * (k.shape[0] / 16 + 64) * F32
    mean_abs = torch.einsum("nh,nhd->hd", p, v.abs())
    codes = (v.abs() / torch.exp2(ev)[..., None]).sum(0)                                      # [heads, hd]
    small = 2.0 ** (-25 - shift) * (p * torch.exp2(ev)).amax(0)[:, None] * codes
    return out, 2.0 ** -8 * out.abs() + rel[:, None] * (mean_abs + out.abs()) + small + 1e-30
