"""Rules on logits before a token is drawn, one logit at a time in fp64 (Python numbers)."""
from __future__ import annotations

import numpy as np


def process(logits, repetition=None, frequency=None, presence=None, history=None, prompt_sets=None, biases=None, allowed_sets=None):
    """logits [R, V]; per row: repetition / frequency / presence numbers, history = list of generated tokens, prompt_sets = set of
    tokens (or None), biases = list of (token, value), allowed_sets = set of tokens (or None: all)."""
    R, V = logits.shape
    out = np.array(logits, dtype=np.float64)
    for r in range(R):
        said = [t for t in (history[r] if history is not None else []) if 0 <= t < V]
        count = {}
        for t in said:
            count[t] = count.get(t, 0) + 1
        prompt = prompt_sets[r] if prompt_sets is not None and prompt_sets[r] is not None else set()
        rep = float(repetition[r]) if repetition is not None else 1.0
        rep = rep if 0 < rep < float("inf") else 1.0
        with np.errstate(invalid="ignore"):
            for t in set(count) | {t for t in prompt if 0 <= t < V}:
                out[r, t] = out[r, t] / rep if out[r, t] > 0 else out[r, t] * rep
            for t, c in count.items():
                out[r, t] -= (float(frequency[r]) if frequency is not None else 0.0) * c + (float(presence[r]) if presence is not None else 0.0)
            for t, v in (biases[r] if biases is not None else []):
                if 0 <= t < V:
                    out[r, t] += v
        if allowed_sets is not None and allowed_sets[r] is not None:
            keep = np.zeros(V, bool)
            keep[[t for t in allowed_sets[r] if 0 <= t < V]] = True
            out[r, ~keep] = -np.inf
    return out


def bitmaps(sets, vocab):
    """[len(sets), ceil(vocab / 32)] uint32: bit t % 32 of word t / 32 = token t."""
    bits = np.zeros((len(sets), (vocab + 31) // 32), np.uint32)
    for m, tokens in enumerate(sets):
        for t in tokens:
            if 0 <= t < vocab:
                bits[m, t // 32] |= np.uint32(1) << np.uint32(t % 32)
    return bits
