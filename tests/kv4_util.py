"""What a cache held in 4 bits stands for, from the definition in 64 bits on the host, and where its bytes lie."""
import math

import torch

# significant bits of a scale, and the exponent of the type's smallest value
SCALES = {torch.float16: (8, -24), torch.bfloat16: (5, -133)}


def scale_of(m, dtype):
    """The smallest value s of `dtype` with few enough significant bits and 7.5 s >= m (m >= 0, finite), one at a time."""
    bits, least = SCALES[dtype]
    if m == 0:
        return 0.0
    power = max(math.frexp(m / 7.5)[1] - bits - 2, least)       # (a few binades too fine, to be sure)
    while True:
        n = math.floor(m / 7.5 / 2.0 ** power) - 1
        while 7.5 * n * 2.0 ** power < m:
            n += 1
        if n <= 2 ** bits:
            return n * 2.0 ** power
        power += 1


def quantise(x):
    """x [..., D] of 16 bits -> (codes [..., D], scales [..., groups], what they stand for [..., D]), float64.  A group with an infinity or a NaN: codes 0,
    scale NaN."""
    D = x.shape[-1]
    rows = x.double().reshape(-1, D)
    groups = (D + 31) // 32
    codes, scales = torch.zeros((rows.shape[0], D), dtype=torch.float64), torch.zeros((rows.shape[0], groups), dtype=torch.float64)
    for g in range(groups):
        part = rows[:, 32 * g:32 * g + 32]
        top = part.abs().amax(1)
        for m in top.unique().tolist():
            if math.isfinite(m):
                scales[top == m, g] = scale_of(m, x.dtype)
        scales[~part.isfinite().all(1), g] = math.nan
        s = scales[:, g:g + 1]
        q = torch.where(s > 0, torch.round(part / s), 0.0).clamp(-7, 7)       # (torch.round: halves to even)
        codes[:, 32 * g:32 * g + 32] = torch.where(s.isnan(), 0.0, q)
    value = codes * scales.repeat_interleave(32, 1)[:, :D]
    return codes.reshape(x.shape), scales.reshape(*x.shape[:-1], groups), value.reshape(x.shape)


def places(slots, page_size, heads, D):
    """For slots [n]: byte addresses within all pages (back to back) of the codes of keys and of values [n, heads, D], which of them are a byte's
    second code, and of the groups' scales [n, heads, groups]."""
    S = (D + 31) // 32
    record = 576 * S
    page_bytes = heads * (page_size // 16) * record
    n, h, d, g = slots[:, None, None], torch.arange(heads)[None, :, None], torch.arange(D)[None, None], torch.arange(S)[None, None]
    base = n // page_size * page_bytes + (h * (page_size // 16) + n % page_size // 16) * record
    token = n % 16
    t, a, i = d // 32, d % 32 // 8, d % 8
    keys = base + (a * 16 + token) * 4 * S + 4 * t + i % 4
    values = base + 256 * S + (token // 4 * 16 + d % 16) * 4 * S + 4 * (d // 32) + token % 4
    scales = base + 512 * S + (token // 4 * S + g) * 8 + token % 4 * 2
    return keys, (i >= 4).expand(keys.shape), values, (d % 32 >= 16).expand(values.shape), scales, scales + 32 * S
