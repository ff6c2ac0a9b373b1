"""Plain implementations, on the CPU and in 64 bits, of the calls over the paged cache of 16 or 8 bits, written from the definitions in the
header: loops over sequences, heads and tokens.  The numbers of e4m3 codes come from the format's definition."""
import math

import numpy as np
import torch

LOWEST = -117
LAST = {torch.float16: 8, torch.bfloat16: 120}                  # e from which on 256 2^e is beyond the type


def _numbers():
    out = np.empty(256)
    for c in range(256):
        power, mantissa = (c >> 3) & 15, c & 7
        size = (1 + mantissa / 8) * 2.0 ** (power - 7) if power else mantissa / 8 * 2.0 ** -6
        size = math.nan if c & 127 == 127 else size
        out[c] = -size if c & 128 else size
    return out


NUMBERS = _numbers()
_POSITIVE = NUMBERS[:127]                                       # ascending


def code_row(x):
    """(codes [128], byte) of one row of fp16 or bf16."""
    f = x.double().numpy()
    if not np.isfinite(f).all():
        return np.full(128, 127, dtype=np.uint8), 255
    top = np.abs(f).max()
    e = LOWEST
    while top > 448 * 2.0 ** e:
        e += 1
    y = np.abs(f) / 2.0 ** e
    hi = np.searchsorted(_POSITIVE, y)                          # the first code that is not below
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - y, y - _POSITIVE[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    if e >= LAST[x.dtype]:
        c = np.minimum(c, np.searchsorted(_POSITIVE, 240.0))
    return (c + 128 * np.signbit(f)).astype(np.uint8), e + 127


def values(codes, scales):
    """64-bit numbers of rows codes [.., 128], scales [..]."""
    x = torch.from_numpy(NUMBERS)[codes.long()]
    return x * torch.exp2(scales.double() - 127)[..., None]


def visible(L, n, i):
    """Keys that new token i of n sees in a sequence of L."""
    return max(L - n + i + 1, 0)
