"""How far the outputs of the calls around the smaller paged caches may be from 64 bits, close to what their arithmetic loses.

Roundings of different terms are independent, so that a sum's error goes by the square root of the sum of squares of its terms' errors.  A rounding to fp32 is
off by at most 2^-24 of its result, one to a type by half a step; sums take three times the largest error of a term as its deviation (five deviations of a
rounding that is equally likely everywhere, where an output is one of some 10^5), and `_SUM` times sqrt(additions) 2^-24 of their terms' sizes."""
import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
_SUM = 8


def softmax_parts(x, v):
    """Weights p, outputs p v, and of each output the root of sum p^2 v^2 and the sum of p |v|."""
    p = torch.softmax(x, -1)
    return p, p @ v, (p.square() @ v.square()).sqrt(), p @ v.abs()


def bound(dtype, x, v, dx, part, extra=0.0):
    """(exact output, its bound) of rows x [heads, keys] of logits, values v [keys, d]; dx: a logit's error; part: a weight's, relative; extra: another summand.

    A weight is e^{x - m}: the logit's error, the rounding of x - m in units of log2 and that of its result, 2^-22 of the exponential (an instruction that is good to
    one unit in the last place, and one rounding more).  A weight enters numerator and denominator, so that its error moves the output by p (v - out): within p (|v| + |out|)."""
    p, out, spread, size = softmax_parts(x, v)
    top = x[torch.isfinite(x)].abs().max()
    weight = dx + 2.0 ** -23 * top + 2.0 ** -22 + part
    own = p.square().sum(-1, keepdim=True).sqrt() * out.abs()
    keys = x.shape[-1]
    sums = _SUM * 2.0 ** -24 * (keys / 32 + 16) ** 0.5 * (size + out.abs())
    return out, HALF_STEP[dtype] * 1.01 * out.abs() + 3 * weight * (spread + own) + sums + extra + 2.0 ** -25


def nibble(dtype, q, k, v, sk, sv, scale):
    """4-bit attention: q [heads, 128], k, v [keys, 128] as the codes stand for them, sk, sv [keys]: the largest scale of a row.

    A score is sum s sum q (16 + c) + sum (l - 16 s) sum q: some 160 additions of partial sums of at most 31 s sum |q| and 16 s + |l| times sum |q|, of 47 s sum |q| + |l| sum |q|
    together, the root of 128 smaller where the q have both signs; l is within |k| + 15 s.  A weight times a scale is two numbers of bf16, off by 2^-16 of itself, and multiplied by 16 + c <= 31; the sums over 16 + c and
    over l - 16 s, whose 16 s cancel, carry fp32 roundings of 47 s + |l|."""
    x = scale * (q @ k.t())
    dx = _SUM * 160 ** 0.5 * 2.0 ** -24 * abs(scale) * float(q.abs().sum(-1).max()) * float((62 * sk + k.abs().amax(-1)).max()) / 128 ** 0.5
    p = torch.softmax(x, -1)
    coded = 3 * 2.0 ** -16 * 31 * (p.square() @ sv.square()).sqrt() + _SUM * 2.0 ** -24 * (len(k) / 32 + 16) ** 0.5 * 62 * (p @ sv)
    return bound(dtype, x, v, dx, 0.0, coded[:, None])


def latent(dtype, parts, q, k, v, scale, visible=None):
    """Attention over latent rows or a prompt's own keys: scores are fp32 sums of exact products, 32 at a time, whose partial sums stay within |q| |k|; a weight enters as `parts` numbers of the type."""
    x = scale * (q @ k.t())
    if visible is not None:
        x = torch.where(visible, x, float("-inf"))
    dx = _SUM * 2.0 ** -24 * abs(scale) * float(q.norm(dim=-1).max() * k.norm(dim=-1).max())
    half = HALF_STEP[dtype]
    return bound(dtype, x, v, dx, half if parts == 1 else half * half)
