"""4-bit pages and page tables in numpy: blocks of 32 channels as a power of two and 4-bit floating-point numbers, rows by
slot.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import functools
from fractions import Fraction

import numpy as np

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # codes 0 to 7; 8 to 15 are their negatives
LOWEST = {"fp16": -23, "bf16": -125}


@functools.lru_cache(maxsize=None)
def _code(x: float, negative: bool, e: int) -> int:
    """The nearest code of x / 2^e, of two as near the even one, in exact rationals.  (0 and -0 are the same key: the sign is its own.)"""
    a = abs(Fraction(x)) / Fraction(2) ** e
    best = min(range(8), key=lambda i: (abs(Fraction(GRID[i]) - a), i % 2))
    return best + (8 if negative else 0)


def encode_block(x, dtype: str):
    """x: 32 numbers of the type -> (32 codes, scale byte); a non-finite number makes the block NaN (codes 0, scale 255)."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return [0] * 32, 255
    top = float(np.abs(x).max())
    e = LOWEST[dtype] if top == 0 else max(LOWEST[dtype], int(np.frexp(top)[1]) - 1 - 2)
    return [_code(float(v), bool(np.signbit(v)), e) for v in x], e + 127


def encode_row(x, dtype: str):
    """128 numbers -> uint8 [64] (channel 2 i in the low half of byte i), uint8 [4]."""
    codes, scales = [], []
    for u in range(4):
        c, s = encode_block(x[32 * u:32 * u + 32], dtype)
        codes += c
        scales.append(s)
    c = np.array(codes, np.uint8)
    return c[0::2] | (c[1::2] << 4), np.array(scales, np.uint8)


def decode_rows(codes, scales):
    """uint8 [..., 64], [..., 4] -> float64 [..., 128]."""
    codes, scales = np.asarray(codes), np.asarray(scales).astype(np.int64)
    grid = np.array(GRID + tuple(-g for g in GRID))
    out = np.empty((*codes.shape[:-1], 128))
    out[..., 0::2], out[..., 1::2] = grid[codes & 15], grid[codes >> 4]
    two = np.where(scales == 255, np.nan, np.ldexp(1.0, scales - 127))
    return out * np.repeat(two, 32, axis=-1)


def split_page(page, page_size: int):
    """uint8 [..., 68 page_size] -> codes [..., page_size, 64], scales [..., page_size, 4]."""
    page = np.asarray(page)
    return (page[..., :64 * page_size].reshape(*page.shape[:-1], page_size, 64),
            page[..., 64 * page_size:].reshape(*page.shape[:-1], page_size, 4))


def rows_of(pages, page_size: int, slots):
    """pages: [n_pages, Hkv, page_size, 128] numbers, or uint8 [n_pages, Hkv, 68 page_size]; slots -> float64 [T, Hkv, 128], zeros
    where a slot is outside."""
    pages = np.asarray(pages)
    if pages.dtype == np.uint8:
        pages = decode_rows(*split_page(pages, page_size))
    out = np.zeros((len(slots), pages.shape[1], 128))
    for t, s in enumerate(slots):
        if 0 <= s < pages.shape[0] * page_size:
            out[t] = pages[s // page_size, :, s % page_size]
    return out


def sequence_slots(table_row, n: int, page_size: int):
    """Slots of a sequence's n tokens."""
    t = np.arange(n)
    return np.asarray(table_row)[t // page_size].astype(np.int64) * page_size + t % page_size
