"""Page tables and slot maps from request lengths: the plain sequential definition (a Python loop in sample order)."""
from __future__ import annotations

import numpy as np

PAGE = 16


def _pages(tokens: int) -> int:
    return (tokens + PAGE - 1) // PAGE


def build(seq_lens, reserve_lens, free_pages, free_count, num_entries, max_tokens):
    """Lists from scratch.  Returns a dict of the outputs and the list of refused samples."""
    seq = [int(x) for x in seq_lens]
    reserve = seq if reserve_lens is None else [int(x) for x in reserve_lens]
    indptr = [0]
    for r in reserve:
        indptr.append(indptr[-1] + _pages(max(r, 0)))
    room = [indptr[s + 1] <= num_entries for s in range(len(seq))]
    cut = [min(x, num_entries) for x in indptr]
    fits = [0 <= seq[s] <= reserve[s] and room[s] for s in range(len(seq))]
    out = _assign([0] * len(seq), seq, fits, cut, np.full(num_entries, -1, np.int64), free_pages, free_count, max_tokens)
    out["page_indptr"] = np.asarray(cut, np.int32)
    return out


def extend(held_lens, new_lens, max_lens, free_pages, free_count, page_indptr, page_indices, max_tokens):
    """More tokens for lists that exist."""
    held, new = [int(x) for x in held_lens], [int(x) for x in new_lens]
    indptr = [int(x) for x in page_indptr]
    fits = []
    for s in range(len(held)):
        end = held[s] + max(new[s], 0)
        ok = held[s] >= 0 and new[s] >= 0
        if ok and new[s] > 0:
            ok = end <= (2 ** 31 - 1 if max_lens is None else int(max_lens[s])) and _pages(end) <= indptr[s + 1] - indptr[s]
            if ok and held[s] % PAGE:
                ok = int(page_indices[indptr[s] + held[s] // PAGE]) >= 0
        fits.append(ok)
    return _assign(held, new, fits, indptr, np.asarray(page_indices).astype(np.int64), free_pages, free_count, max_tokens)


def _assign(held, new, fits, indptr, indices, free_pages, free_count, max_tokens):
    left, dry, at = max(int(free_count), 0), False, 0
    tokens, slots, lens, refused = [0], np.full(max_tokens, -1, np.int64), [], []
    for s in range(len(held)):
        count = max(new[s], 0)
        end = held[s] + count
        ok = fits[s] and at + count <= max_tokens
        need = list(range(_pages(held[s]), _pages(end))) if ok else []
        if need and (dry or len(need) > left):
            ok, dry, need = False, True, []
        for j in need:
            left -= 1
            indices[indptr[s] + j] = int(free_pages[left])
        if ok:
            for i in range(count):
                pos = held[s] + i
                slots[at + i] = indices[indptr[s] + pos // PAGE] * PAGE + pos % PAGE
        else:
            refused.append(s)
        lens.append(end if ok else held[s])
        at += count
        tokens.append(min(at, max_tokens))
    return dict(page_indices=indices.astype(np.int32), token_indptr=np.asarray(tokens, np.int32), slot_map=slots,
                lens_out=np.asarray(lens, np.int32), free_count=left, refused=refused)
