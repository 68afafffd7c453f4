"""Pins of the oracle for rules on logits (by hand) and the library's refusals that need no device."""
import ctypes

import numpy as np
import pytest

from oracle import logits_rules as lr


def test_by_hand():
    x = np.array([[2.0, -2.0, 0.0, 1.0, 4.0, -1.0]])
    out = lr.process(x, repetition=[2.0], frequency=[0.5], presence=[0.25], history=[[0, 1, 1, 9, -3]], prompt_sets=[{4, 2}],
                     biases=[[(3, 1.5), (3, -1.0), (0, 0.125), (77, 5.0)]], allowed_sets=[{0, 1, 3, 4}])
    # 0: 2/2 - .5 - .25 + .125;  1: -4 - 1 - .25;  2: masked;  3: 1 + .5;  4: 4/2 (prompt only: no count);  5: masked
    assert out.tolist() == [[0.375, -5.25, -np.inf, 1.5, 2.0, -np.inf]]


def test_nothing_to_do_and_nothing_left():
    x = np.array([[1.0, -3.0]])
    assert lr.process(x).tolist() == x.tolist()
    assert lr.process(x, repetition=[0.0], history=[[0, 1]]).tolist() == x.tolist()      # not a penalty
    assert lr.process(x, repetition=[float("nan")], history=[[0]]).tolist() == x.tolist()
    assert np.isneginf(lr.process(x, allowed_sets=[set()])).all()


def test_bitmaps_by_hand():
    assert lr.bitmaps([[0, 31, 32, 40, -1], []], 40).tolist() == [[(1 << 31) + 1, 1], [0, 0]]


FAKE = 1 << 20


def test_host_refusals():
    import paper_2502_02534_b200 as psa
    from paper_2502_02534_b200.binding import _LogitsRules
    lib = psa.library()

    def call(rules=None, logits=FAKE, code=0, stride=104, rows=2, vocab=100, out=FAKE + 4096, out_code=0, out_stride=104):
        r = _LogitsRules(**(rules or {}))
        return lib.psa_process_logits(logits, code, stride, rows, vocab, ctypes.byref(r), out, out_code, out_stride, None)
    assert call(rows=-1) == 1 and call(vocab=-1) == 1 and call(vocab=0) == 1 and call(rows=0) == 0
    assert call(rows=65536) == 2 and call(vocab=(1 << 24) + 1, stride=1 << 25, out_stride=1 << 25) == 2 and call(code=2) == 2 and call(out_code=-1) == 2
    assert call(logits=None) == 1 and call(out=None) == 1 and call(logits=FAKE + 8) == 1 and call(out=FAKE + 2) == 1
    assert call(stride=96) == 1 and call(stride=101) == 1 and call(out_stride=100) == 1
    assert call(out=FAKE, out_code=1) == 1 and call(out=FAKE, out_stride=112) == 1                 # in place, but not the same array
    # shifted by a row or by less than a row (bf16: 208 bytes from row to row, 200 of them used), either way round, and f32 into the end of them
    assert call(out=FAKE + 208) == 1 and call(out=FAKE + 16) == 1 and call(out=FAKE - 208) == 1 and call(out=FAKE - 16) == 1
    assert call(out=FAKE + 400, out_code=1) == 1 and call(out=FAKE + 720, stride=408, out_stride=408) == 1
    assert call(dict(history=FAKE)) == 1 and call(dict(history=FAKE, history_lens=FAKE, history_capacity=8, history_stride=4)) == 1
    assert call(dict(bias_indptr=FAKE, num_biases=3)) == 1 and call(dict(num_biases=-1)) == 1
    assert call(dict(prompt_bits=FAKE, prompt_row_words=3)) == 1 and call(dict(mask_bits=FAKE, mask_row_words=3)) == 1
    assert lib.psa_process_logits(FAKE, 0, 104, 2, 100, None, FAKE, 0, 104, None) == 1

    def mark(ids=FAKE, n=4, indptr=FAKE, rows=2, vocab=100, bits=FAKE, words=4):
        return lib.psa_mark_tokens(ids, n, indptr, rows, vocab, bits, words, None)
    assert mark(n=-1) == 1 and mark(rows=-1) == 1 and mark(vocab=0) == 1 and mark(rows=0) == 0 and mark(rows=65536) == 2 and mark(vocab=(1 << 24) + 1) == 2
    assert mark(ids=None) == 1 and mark(indptr=None) == 1 and mark(bits=None) == 1 and mark(words=3) == 1


def test_binding_refusals():
    import torch
    import paper_2502_02534_b200 as psa
    x = torch.zeros((2, 104))[:, :100]
    i = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    for kw, match in ((dict(), "current CUDA device"), (dict(out=torch.zeros((2, 99))), "same shape"), (dict(out=x.half()), "bf16 or f32"),
                      (dict(history=i(2, 4)), "go together"), (dict(history=i(1, 4), history_lens=i(2)), "history"),
                      (dict(bias_indptr=i(3)), "go together"), (dict(prompt_rows=i(2)), "without"), (dict(mask_bits=i(2, 3)), "words"),
                      (dict(mask_bits=i(1, 4)), "one bitmap per row"), (dict(prompt_bits=i(4, 8)[:, ::2]), "contiguous")):
        with pytest.raises(ValueError, match=match):
            psa.process_logits(x, **kw)
    with pytest.raises(ValueError, match="bf16 or f32"):
        psa.process_logits(x.half())
    with pytest.raises(ValueError, match="vocabulary"):
        psa.process_logits(torch.zeros((2, 208))[:, ::2])
    with pytest.raises(ValueError, match="current CUDA device"):
        psa.mark_tokens(i(4), i(3), 100)
    with pytest.raises(ValueError, match="words"):
        psa.mark_tokens(i(4), i(3), 100, i(2, 3))
    with pytest.raises(ValueError, match="rows"):
        psa.mark_tokens(i(4), i(0), 100)
