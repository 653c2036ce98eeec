"""The 4-bit paged KV cache and block tables, by their definitions.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A value is ``(-1)^s * magnitude * 2^(b - 127)`` with magnitudes 0, .5, 1, 1.5, 2,
3, 4, 6 (codes 0-7, sign in bit 3) and a byte ``b`` that 32 consecutive dims of
a key share.  Stored rows take the smallest exponent ``e = b - 127`` within
``[-125, 125]`` under which no magnitude of the 32 exceeds ``7 * 2^e``, and the
nearest code, ties to the even one; infinities take the largest magnitude and
NaN code 0.  A record (one page and KV head) is a list of nibbles, the lower
one of a byte first, then the scale bytes; positions by key and dim are below.
"""
from __future__ import annotations

import numpy as np

from .append import append_targets

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
PAGE = 16


def kv4_round(x):
    """Codes ``[..., d]`` and scale bytes ``[..., d / 32]`` of float values."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(-1, 32)
    codes = np.zeros(blocks.shape, dtype=np.uint8)
    scales = np.zeros(len(blocks), dtype=np.uint8)
    for i, v in enumerate(blocks):
        nan = np.isnan(v)
        v = np.where(nan, 0.0, v)
        top = np.abs(v).max()
        e = -125
        while e < 125 and top > 7.0 * 2.0 ** e:
            e += 1
        scales[i] = e + 127
        y = np.minimum(np.abs(v) / 2.0 ** e, 6.0)
        off = np.abs(y[:, None] - MAGNITUDES)
        near = off == off.min(axis=1, keepdims=True)
        pick = np.array([min(np.nonzero(row)[0], key=lambda c: (c % 2, c)) for row in near])
        codes[i] = np.where(nan, 0, pick + 8 * np.signbit(v))
    return codes.reshape(x.shape), scales.reshape(*x.shape[:-1], x.shape[-1] // 32)


def kv4_values(codes, scales):
    """The values that codes and scale bytes stand for."""
    size = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return size * np.repeat(2.0 ** (scales.astype(np.float64) - 127.0), 32, axis=-1)


def nibble_at(which, d):
    """``[16, d]``: the nibble of a ``which`` ("k" or "v") record that holds (key, dim)."""
    out = np.zeros((PAGE, d), dtype=np.int64)
    for key in range(PAGE):
        for dim in range(d):
            if which == "k":  # [4][16 keys][d / 4 nibbles]
                piece, inside = divmod(dim, d // 4)
                out[key, dim] = (piece * PAGE + key) * (d // 4) + inside
            else:  # [4 key groups][16][4 keys][d / 16 nibbles]
                piece, inside = divmod(dim, d // 16)
                out[key, dim] = ((key // 4 * 16 + piece) * 4 + key % 4) * (d // 16) + inside
    return out


def scale_at(d):
    """``[16, d / 32]``: the byte of a record that holds the scale of (key, block)."""
    return 8 * d + np.arange(d // 32)[None, :] * PAGE + np.arange(PAGE)[:, None]


def kv4_read(which, pages, d):
    """A pool ``[P, Hkv, 17 d / 2]`` as codes ``[P, 16, Hkv, d]`` and scale bytes ``[P, 16, Hkv, d / 32]``."""
    nib = nibble_at(which, d)
    codes = (pages[:, :, nib // 2] >> (4 * (nib % 2)).astype(np.uint8)) & 15
    return codes.transpose(0, 2, 1, 3), pages[:, :, scale_at(d)].transpose(0, 2, 1, 3)


def kv4_write(which, pages, page, slot, codes, scales):
    """Write one key's codes ``[Hkv, d]`` and scale bytes into a pool, in place."""
    d = codes.shape[-1]
    for dim, nib in enumerate(nibble_at(which, d)[slot]):
        byte, shift = nib // 2, 4 * (nib % 2)
        keep = pages[page, :, byte] & (0xF0 >> shift)
        pages[page, :, byte] = keep | (codes[:, dim] << shift)
    for block, byte in enumerate(scale_at(d)[slot]):
        pages[page, :, byte] = scales[:, block]


def kv4_append(batch, k_new, v_new, k_pages, v_pages):
    """New 4-bit pools with the step's rows written in."""
    out = []
    for which, new, pages in (("k", k_new, k_pages), ("v", v_new, v_pages)):
        pages = np.array(pages, copy=True)
        codes, scales = kv4_round(new)
        for row, page, slot in append_targets(batch):
            kv4_write(which, pages, page, slot, codes[row], scales[row])
        out.append(pages)
    return tuple(out)


def block_tables(seqs, free_pages, table, num_pages):
    """The step's block table, flat slots by packed row (a dict) and pages taken."""
    table = np.array(table, copy=True)
    slots, at = {}, 0
    for r, (q_len, kv_len, q_start) in enumerate(np.asarray(seqs, dtype=np.int64).reshape(-1, 3)):
        for pos in range(kv_len - q_len, kv_len):
            if pos % PAGE == 0:
                page = int(free_pages[at])
                table[r, pos // PAGE] = page if 0 <= page < num_pages else -1
                at += 1
            page = int(table[r, pos // PAGE])
            slots[int(q_start + pos - (kv_len - q_len))] = page * PAGE + pos % PAGE if 0 <= page < num_pages else -1
    return table, slots, at
