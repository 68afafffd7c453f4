"""What the operators over a paged bf16 cache and the log probabilities refuse: on the host, before anything is launched."""
import ctypes

import pytest

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def tensors(**change):
    import torch
    bf, i32 = torch.bfloat16, torch.int32
    d = dict(q=torch.zeros(6, 8, 64, dtype=bf), k=torch.zeros(9, 2, 16, 64, dtype=bf), v=torch.zeros(9, 2, 16, 64, dtype=bf), indptr=torch.zeros(4, dtype=i32),
             indices=torch.zeros(9, dtype=i32), lens=torch.zeros(3, dtype=i32), q_indptr=torch.zeros(4, dtype=i32), lse=torch.zeros(6, 8), w=torch.zeros(9, 2, 16),
             slots=torch.zeros(6, dtype=torch.int64), new=torch.zeros(6, 2, 64, dtype=bf), free=torch.zeros(9, dtype=i32), count=torch.zeros(1, dtype=i32),
             budgets=torch.zeros(3, dtype=i32), logits=torch.zeros(4, 104)[:, :100], tokens=torch.zeros(4, dtype=i32))
    d.update(change)
    return d


def attend(d, **kw):
    from paper_2502_02534_b200 import attend_paged
    attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], **kw)


def weights(d, **kw):
    from paper_2502_02534_b200 import accumulate_weights
    accumulate_weights(d["q"], d["lse"], d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], d["w"], **kw)


def store(d, **kw):
    from paper_2502_02534_b200 import store_kv
    store_kv(d["new"], d["new"].clone(), d["slots"], d["k"], d["v"], **kw)


def evict(d, recent=1, **kw):
    from paper_2502_02534_b200 import evict_pages
    evict_pages(d["w"], d["indptr"], d["indices"], d["lens"], d["budgets"], recent, d["free"], d["count"], **kw)


def logprobs(d, top=3, **kw):
    from paper_2502_02534_b200 import token_logprobs
    token_logprobs(d["logits"], d["tokens"], top, **kw)


@pytest.mark.parametrize("call", [attend, weights, store, evict, logprobs])
def test_tensors_have_to_be_on_the_gpu(call):
    with pytest.raises(ValueError, match="current CUDA device"):
        call(tensors())


def test_tensors_of_the_wrong_kind():
    import torch
    z = torch.zeros
    bf, i32 = torch.bfloat16, torch.int32
    bad = [
        (attend, dict(q=z(6, 8, 64)), "bf16"), (attend, dict(q=z(48, 64, dtype=bf)), "tokens, heads, head_dim"), (attend, dict(k=z(9, 2, 8, 64, dtype=bf)), "k_pool"),
        (attend, dict(v=z(8, 2, 16, 64, dtype=bf)), "same shape"), (attend, dict(v=z(9, 16, 2, 64, dtype=bf).transpose(1, 2)), "same shape and strides"),
        (attend, dict(indptr=z(3, dtype=i32)), "page_indptr"), (attend, dict(lens=z(3, dtype=torch.int64)), "kv_lens"), (attend, dict(q_indptr=z(3, dtype=i32)), "q_indptr"),
        (attend, dict(q_indptr=None), "one row"), (attend, dict(q=z(64, 6, 8, dtype=bf).permute(1, 2, 0)), "contiguous last"), (weights, dict(w=z(9, 2, 8)), "weights"),
        (weights, dict(w=z(9, 2, 16, dtype=torch.float64)), "weights"), (weights, dict(lse=z(5, 8)), "lse"), (store, dict(slots=z(5, dtype=torch.int64)), "slot_map"),
        (store, dict(slots=z(6, dtype=i32)), "slot_map"), (store, dict(new=z(6, 3, 64, dtype=bf)), "k_pool"), (evict, dict(w=z(9, 32)), "weights"),
        (evict, dict(budgets=z(2, dtype=i32)), "budgets"), (evict, dict(free=z(9)), "free_pages"), (logprobs, dict(logits=z(4, 100, dtype=torch.float64)), "bf16 or f32"),
        (logprobs, dict(logits=z(100)), "rows, vocab|out of range|index"), (logprobs, dict(tokens=z(3, dtype=i32)), "tokens"), (logprobs, dict(logits=z(100, 4).t()), "contiguous"),
    ]
    for call, change, match in bad:
        with pytest.raises((ValueError, IndexError), match=match):
            call(tensors(**change))
    d = tensors()
    for call, kw, match in ((attend, dict(out=z(6, 8, 32, dtype=bf)), "out"), (attend, dict(out=z(6, 8, 64, dtype=torch.float16)), "bf16 or f32"),
                            (attend, dict(prior_lse=z(6, 8)), "go together"), (attend, dict(prior_out=z(6, 4, 64), prior_lse=z(6, 8)), "prior_out"),
                            (attend, dict(status=z(1)), "status"), (weights, dict(weights_out=z(9, 2, 4)), "weights_out"), (evict, dict(recent=0), "recent"),
                            (evict, dict(lens_out=z(2, dtype=i32)), "lens_out"), (evict, dict(page_indices_out=z(3, dtype=i32)), "page_indices_out"),
                            (logprobs, dict(top_ids=z(4, 2, dtype=i32)), "top_ids"), (logprobs, dict(temperature=z(3)), "temperature"), (logprobs, dict(top=-1), "negative")):
        with pytest.raises((ValueError, RuntimeError), match=match):
            call(d, **kw)


class Library:
    """The C entry points with arguments that pass, of which some are changed; pointers that are never followed."""
    P = 1 << 20

    def strides(self, *v):
        return (ctypes.c_int64 * len(v))(*v)

    def attend(self, **c):
        from paper_2502_02534_b200 import library
        a = dict(q=self.P, qs=self.strides(512, 64), qi=self.P, T=6, B=3, Hq=8, Hkv=2, D=64, scale=0.125, k=self.P, v=self.P, ps=self.strides(2048, 1024, 64), pages=9,
                 indptr=self.P, indices=self.P, entries=9, lens=self.P, po=None, pd=0, pl=None, out=self.P, od=0, lse=self.P, status=None, scratch=None, bytes=0)
        a.update(c)
        return library().psa_attend_paged(*[a[k] for k in ("q", "qs", "qi", "T", "B", "Hq", "Hkv", "D", "scale", "k", "v", "ps", "pages", "indptr", "indices", "entries",
                                                          "lens", "po", "pd", "pl", "out", "od", "lse", "status", "scratch", "bytes")], None)

    def weights(self, **c):
        from paper_2502_02534_b200 import library
        a = dict(q=self.P, qs=self.strides(512, 64), qi=self.P, T=6, B=3, Hq=8, Hkv=2, D=64, scale=0.125, lse=self.P, k=self.P, ps=self.strides(2048, 1024, 64), pages=9,
                 indptr=self.P, indices=self.P, entries=9, lens=self.P, w=self.P, wo=self.P, status=None, scratch=None, bytes=0)
        a.update(c)
        return library().psa_accumulate_weights(*[a[k] for k in ("q", "qs", "qi", "T", "B", "Hq", "Hkv", "D", "scale", "lse", "k", "ps", "pages", "indptr", "indices",
                                                                "entries", "lens", "w", "wo", "status", "scratch", "bytes")], None)

    def store(self, **c):
        from paper_2502_02534_b200 import library
        a = dict(k=self.P, v=self.P, s=self.strides(128, 64), slots=self.P, T=6, Hkv=2, D=64, kp=self.P, vp=self.P, ps=self.strides(2048, 1024, 64), pages=9, status=None)
        a.update(c)
        return library().psa_store_kv(*[a[k] for k in ("k", "v", "s", "slots", "T", "Hkv", "D", "kp", "vp", "ps", "pages", "status")], None)

    def evict(self, **c):
        from paper_2502_02534_b200 import library
        a = dict(w=self.P, pages=9, Hkv=2, indptr=self.P, indices=self.P, entries=9, lens=self.P, budgets=self.P, B=3, recent=1, free=self.P, cap=9, count=self.P,
                 io=self.P, lo=self.P, co=self.P, status=None, scratch=None, bytes=0)
        a.update(c)
        return library().psa_evict_pages(*[a[k] for k in ("w", "pages", "Hkv", "indptr", "indices", "entries", "lens", "budgets", "B", "recent", "free", "cap", "count",
                                                         "io", "lo", "co", "status", "scratch", "bytes")], None)

    def logprobs(self, **c):
        from paper_2502_02534_b200 import library
        a = dict(x=self.P, dt=1, stride=104, R=4, V=100, tok=self.P, temp=None, lp=self.P, h=self.P, top=3, ids=self.P, tops=self.P, ts=3)
        a.update(c)
        return library().psa_token_logprobs(*[a[k] for k in ("x", "dt", "stride", "R", "V", "tok", "temp", "lp", "h", "top", "ids", "tops", "ts")], None)


def test_the_library_refuses():
    c = Library()
    s = c.strides
    for call, change, want in [
        (c.attend, dict(D=96), UNSUPPORTED), (c.attend, dict(Hq=6), UNSUPPORTED), (c.attend, dict(Hq=32), UNSUPPORTED), (c.attend, dict(Hq=7), UNSUPPORTED),
        (c.attend, dict(T=-1), INVALID), (c.attend, dict(B=1 << 21), UNSUPPORTED), (c.attend, dict(T=1 << 25), UNSUPPORTED), (c.attend, dict(Hkv=0), INVALID),
        (c.attend, dict(q=c.P + 8), INVALID), (c.attend, dict(k=c.P + 8), INVALID), (c.attend, dict(v=c.P + 2), INVALID), (c.attend, dict(out=c.P + 4), INVALID),
        (c.attend, dict(qs=s(512, 60)), INVALID), (c.attend, dict(qs=s(0, 64)), INVALID), (c.attend, dict(ps=s(2048, 1024, 63)), INVALID),
        (c.attend, dict(ps=s(2048, -1024, 64)), INVALID), (c.attend, dict(qi=None), INVALID), (c.attend, dict(lens=None), INVALID), (c.attend, dict(scale=0.0), INVALID),
        (c.attend, dict(scale=float("nan")), INVALID), (c.attend, dict(od=2), UNSUPPORTED), (c.attend, dict(po=c.P), INVALID), (c.attend, dict(pl=c.P), INVALID),
        (c.attend, dict(po=c.P, pl=c.P, pd=1), INVALID), (c.attend, dict(status=c.P + 2), INVALID), (c.attend, dict(pages=0), INVALID),
        (c.attend, dict(pages=1 << 40), UNSUPPORTED), (c.attend, {}, WORKSPACE), (c.attend, dict(scratch=c.P, bytes=100), WORKSPACE),
        (c.attend, dict(scratch=c.P + 16, bytes=1 << 40), WORKSPACE), (c.attend, dict(T=0), 0), (c.attend, dict(B=0), 0),
        (c.weights, dict(D=32), UNSUPPORTED), (c.weights, dict(lse=None), INVALID), (c.weights, dict(w=None), INVALID), (c.weights, dict(wo=c.P + 2), INVALID),
        (c.weights, dict(scale=-1.0), INVALID), (c.weights, {}, WORKSPACE), (c.weights, dict(T=0), 0),
        (c.store, dict(D=32), UNSUPPORTED), (c.store, dict(T=-1), INVALID), (c.store, dict(k=c.P + 8), INVALID), (c.store, dict(s=s(128, 60)), INVALID),
        (c.store, dict(ps=s(2048, 1020, 64)), INVALID), (c.store, dict(slots=None), INVALID), (c.store, dict(kp=None), INVALID), (c.store, dict(T=1 << 31), UNSUPPORTED),
        (c.store, dict(slots=c.P + 4), INVALID), (c.store, dict(T=0), 0),
        (c.evict, dict(recent=0), INVALID), (c.evict, dict(w=c.P + 4), INVALID), (c.evict, dict(count=None), INVALID), (c.evict, dict(B=1 << 21), UNSUPPORTED),
        (c.evict, dict(entries=-1), INVALID), (c.evict, dict(lens=None), INVALID), (c.evict, {}, WORKSPACE),
        (c.logprobs, dict(dt=3), UNSUPPORTED), (c.logprobs, dict(V=0), INVALID), (c.logprobs, dict(top=65), UNSUPPORTED), (c.logprobs, dict(V=2, top=3), UNSUPPORTED),
        (c.logprobs, dict(stride=99), INVALID), (c.logprobs, dict(stride=100), INVALID), (c.logprobs, dict(x=c.P + 8), INVALID), (c.logprobs, dict(tok=None), INVALID),
        (c.logprobs, dict(R=65536), UNSUPPORTED), (c.logprobs, dict(ts=2), INVALID), (c.logprobs, dict(V=1 << 25, stride=1 << 25), UNSUPPORTED), (c.logprobs, dict(R=0), 0),
    ]:
        assert call(**change) == want, (call.__name__, change)


def test_scratch_sizes():
    from paper_2502_02534_b200 import library
    lib = library()
    small, large = lib.psa_attend_paged_scratch_bytes(8, 2, 8, 2, 64), lib.psa_attend_paged_scratch_bytes(8192, 2, 64, 8, 128)
    assert 0 < small < large < 64 << 20
    assert lib.psa_attend_paged_scratch_bytes(-1, 2, 8, 2, 64) == lib.psa_attend_paged_scratch_bytes(8, 2, 8, 0, 64) == 0
    assert 0 < lib.psa_accumulate_weights_scratch_bytes(8, 2) < lib.psa_accumulate_weights_scratch_bytes(1 << 20, 2) and lib.psa_accumulate_weights_scratch_bytes(8, -2) == 0
    assert 0 < lib.psa_evict_pages_scratch_bytes(0, 0) < lib.psa_evict_pages_scratch_bytes(10, 1000) and lib.psa_evict_pages_scratch_bytes(1, -1) == 0
