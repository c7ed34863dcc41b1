"""CPU oracle of the 8-bit base cache -- test infrastructure.

Only the tests may import this module; it shares no code with the product.  A row of 128 values
becomes 128 e4m3 codes and one exponent byte b and stands for code * 2^(b - 127); with amax the
largest magnitude among its finite values, E = b - 127 is the smallest integer in [-117, 119] with
amax <= 448 * 2^E; a code is x * 2^-E clamped to +-448, rounded to nearest even; what is not finite
becomes NaN.  Written as a search among the values a code can take, in fp64.

Parity status: pinned in tests/test_fp8_oracle.py (every code is a fixed point, ties and borders by
hand, the exponent's borders, the page layout as a bijection).
"""
from __future__ import annotations

import numpy as np

D, PS = 128, 16
# value of codes 0 .. 126 (3 fraction bits, exponent bias 7); 127 is NaN, + 128 the negative ones
CODE_VALUES = np.array([(c % 8) / 8 * 2.0 ** -6 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7) for c in range(127)])
_MIDS = (CODE_VALUES[1:] + CODE_VALUES[:-1]) / 2


def exponent(x):
    """E of rows x [..., 128]."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=-1)
    limits = np.array([448.0 * 2.0 ** e for e in range(-117, 119)])
    return np.searchsorted(limits, a, side="left") - 117


def codes(x):
    """Codes (0 .. 255) of rows x, and E."""
    x = np.asarray(x, dtype=np.float64)
    e = exponent(x)
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.abs(x) * np.exp2(-e.astype(np.float64))[..., None]
    fine = np.isfinite(x)
    z = np.where(fine, np.minimum(z, 448.0), 0.0)
    c = np.searchsorted(_MIDS, z, side="left")
    tie = (c < 126) & (z == _MIDS[np.minimum(c, 125)])
    c = np.where(tie & (c % 2 == 1), c + 1, c)
    return np.where(fine, c + 128 * np.signbit(x), 127).astype(np.uint8), e


def values(c, e):
    """What codes and exponents stand for."""
    half = np.concatenate([CODE_VALUES, [np.nan]])
    return np.concatenate([half, -half])[c] * np.exp2(e.astype(np.float64))[..., None]


def nearest(x):
    """What the cache holds after rows x were written."""
    return values(*codes(x))


def page_bytes(hkv):
    return 4096 * hkv + -(-32 * hkv // 128) * 128


def k_byte(t, i):
    return (i // 64) * 1024 + (t + 16 * ((i % 16) // 4)) * 16 + 8 * ((i // 32) % 2) + 4 * ((i % 32) // 16) + i % 4


def v_byte(t, i):
    return (i // 64) * 1024 + (i % 16 + 16 * (t // 4)) * 16 + 8 * ((i // 32) % 2) + 4 * ((i // 16) % 2) + t % 4


def write(pool, page, slot, k, v):
    """Rows k and v [hkv][128] (fp64) into slot `slot` of page `page` of pool [pages][page_bytes] (uint8)."""
    hkv = k.shape[0]
    i = np.arange(D)
    for j, (rows, where) in enumerate(((k, k_byte), (v, v_byte))):
        c, e = codes(rows)
        for h in range(hkv):
            pool[page, h * 4096 + j * 2048 + where(slot, i)] = c[h]
            pool[page, hkv * 4096 + h * 32 + j * 16 + slot] = e[h] + 127


def read(pool, page, slot, hkv):
    """K and V [hkv][128] (fp64) that the slot stands for."""
    i, h = np.arange(D)[None], np.arange(hkv)[:, None]
    out = []
    for j, where in enumerate((k_byte, v_byte)):
        e = pool[page, hkv * 4096 + h[:, 0] * 32 + j * 16 + slot].astype(np.int64) - 127
        out.append(values(pool[page, h * 4096 + j * 2048 + where(slot, i)], e))
    return out
