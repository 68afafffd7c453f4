"""Cases that measure the operators for several new tokens at once and for bounded caches: K/V rows stored into a paged cache,
attention of a chunk over it, the weight each cached token received, eviction of pages by that weight, and log probabilities of given
tokens.

``own`` chooses between the plain form (elementary torch operations, this file) and the library's entry points.  Both take
what ``prepare`` makes.  Shapes follow the configurations of ``psa_workloads`` (8 to 256 samples, 2 to 8 KV heads of 64 or 128
channels, answers of up to 4096 tokens, prompts of up to 16384) and the 131072-token vocabulary of the sampling tests.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16          # tokens per page
DEVICE = "cuda"


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # K and V of one new token for each of 32 samples into their pages
        dict(name="store-step", op="store", samples=32, new_lo=1, new=1, kv_heads=8, dim=128),
        # answers or prompt chunks of many lengths into the cache at once
        dict(name="store-turns", op="store", samples=64, new_lo=0, new=2048, kv_heads=8, dim=128),
        # the smallest configuration: 8 samples that take 5 tokens each
        dict(name="attend-small", op="attend", samples=8, new_lo=5, new=5, cached_lo=1, cached=128, q_heads=8, kv_heads=2, dim=64, prior=False),
        # a few drafted tokens of every running sample are verified; what they see of the shared prompt was attended apart
        dict(name="attend-verify", op="attend", samples=64, new_lo=4, new=4, cached_lo=0, cached=4096, q_heads=64, kv_heads=8, dim=128, prior=True),
        # four samples get a new turn each
        dict(name="attend-turns", op="attend", samples=4, new_lo=1, new=512, cached_lo=0, cached=8192, q_heads=32, kv_heads=8, dim=128, prior=False),
        # a chunk of one long prompt
        dict(name="attend-long", op="attend", samples=1, new_lo=4096, new=4096, cached_lo=12288, cached=12288, q_heads=64, kv_heads=8, dim=128,
             prior=False),
        # one decode step's weights, per cached token
        dict(name="weights-step", op="weights", samples=64, new_lo=1, new=1, cached_lo=0, cached=4096, q_heads=64, kv_heads=8, dim=128),
        # the weights that a long chunk gives to what came before it
        dict(name="weights-chunk", op="weights", samples=1, new_lo=2048, new=2048, cached_lo=8192, cached=8192, q_heads=32, kv_heads=8, dim=128),
        # a few short samples over their budget
        dict(name="evict-few", op="evict", samples=8, held_lo=0, held=512, budget=12, recent=4, kv_heads=2),
        # a full batch of answers of up to 8192 tokens, cut to 2048 each
        dict(name="evict-batch", op="evict", samples=256, held_lo=0, held=8192, budget=128, recent=16, kv_heads=8),
        # a few answers' last tokens, small vocabulary
        dict(name="logprobs-few", op="logprobs", rows=8, vocab=3001, top=5, dtype="f32"),
        # a full batch over a large vocabulary
        dict(name="logprobs-batch", op="logprobs", rows=256, vocab=131072, top=20, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["store", "attend", "attend", "attend", "weights", "evict", "logprobs"])
    dim = rng.choice([64, 128])
    if op == "store":
        return dict(op=op, samples=_log_int(rng, 1, 64), new_lo=rng.choice([0, 1]), new=_log_int(rng, 1, 2048), kv_heads=rng.choice([1, 2, 8]), dim=dim)
    if op in ("attend", "weights"):
        kv = rng.choice([1, 2, 8])
        heads = kv * rng.choice([1, 2, 4, 8])
        most = 4096 if op == "attend" else 2048
        new = _log_int(rng, 1, most)
        cached = _log_int(rng, 1, 12288 if op == "attend" else 8192)
        # no more scores than the largest listed case has
        samples = _log_int(rng, 1, max(1, min(64, 64 * most * (most + 8192) // 2 // (heads * new * (new + cached)))))
        case = dict(op=op, samples=samples, new_lo=rng.choice([1, new]), new=new, cached_lo=rng.choice([0, cached // 2]), cached=cached,
                    q_heads=heads, kv_heads=kv, dim=dim)
        if op == "attend":
            case["prior"] = rng.random() < 0.3
        return case
    if op == "evict":
        held = _log_int(rng, 16, 8192)
        budget = _log_int(rng, 1, held // 16)
        return dict(op=op, samples=_log_int(rng, 1, 256), held_lo=rng.choice([0, held // 2]), held=held, budget=budget, recent=rng.randint(1, budget),
                    kv_heads=rng.choice([1, 2, 8]))
    return dict(op=op, rows=_log_int(rng, 1, 256), vocab=_log_int(rng, 100, 131072), top=rng.choice([0, 1, 5, 20, 32]), dtype=rng.choice(["bf16", "bf16", "f32"]))


# ------------------------------------------------------------------------------------------------------------ inputs
def _lengths(rng, n, lo, hi):
    """n whole numbers spread evenly over [lo, hi], in random order."""
    at = (np.arange(n) + rng.random(n)) / n
    return rng.permutation(np.minimum(hi, lo + np.floor((hi - lo + 1) * at))).astype(np.int32)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)


def _normal(gen, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(dtype)


def _scan(a):
    return np.concatenate([[0], np.cumsum(a, dtype=np.int64)])


def _pool_pages(n, lo, hi, more):
    """Pages that hold n samples with _lengths(.., n, lo, hi) tokens and `more` in all, whatever the seed."""
    return (n * lo + (hi - lo + 1) * (n + 1) // 2 + more) // PAGE + n + 32


def _new_lens(case):
    """Tokens each sample gets, the same for every seed: they shape the batch."""
    return _lengths(np.random.default_rng(9), case["samples"], case["new_lo"], case["new"])


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    return {"store": _prepare_store, "attend": _prepare_attend, "weights": _prepare_weights, "evict": _prepare_evict,
            "logprobs": _prepare_logprobs}[case["op"]](case, rng, gen)


def _prepare_store(case, rng, gen):
    new = _new_lens(case)
    pages = (new.astype(np.int64) + PAGE - 1) // PAGE
    total_pages = int(pages.sum()) + 8
    ids = rng.permutation(total_pages)[:int(pages.sum())]
    sample = np.repeat(np.arange(len(new)), new)
    pos = np.arange(len(sample)) - np.repeat(_scan(new)[:-1], new)
    slots = ids[_scan(pages)[sample] + pos // PAGE] * PAGE + pos % PAGE
    slots = np.concatenate([slots, np.full(3, -1)])           # a batch padded to its captured size ends in empty rows
    heads, dim = case["kv_heads"], case["dim"]
    pool = lambda: torch.zeros((total_pages, heads, PAGE, dim), dtype=torch.bfloat16, device=DEVICE)  # noqa: E731
    return dict(case=case, slots=torch.from_numpy(slots.astype(np.int64)).to(DEVICE), k=_normal(gen, (len(slots), heads, dim)),
                v=_normal(gen, (len(slots), heads, dim)), pool_k=pool(), pool_v=pool())


def _paged(case, rng, gen):
    """Samples that hold cached tokens and as many new ones as _new_lens says, their pages scattered over the pool."""
    n, hkv, dim = case["samples"], case["kv_heads"], case["dim"]
    new = _new_lens(case)
    lens = new + _lengths(rng, n, case["cached_lo"], case["cached"])
    pages = (lens + PAGE - 1) // PAGE
    indptr = _scan(pages)
    total_pages = _pool_pages(n, case["cached_lo"], case["cached"], int(new.sum()))
    indices = rng.permutation(total_pages)[:int(indptr[-1])]
    q_indptr = _scan(new)
    tokens = int(q_indptr[-1])
    return dict(case=case, kv_lens=_i32(lens), page_indptr=_i32(indptr), page_indices=_i32(indices), q_indptr=_i32(q_indptr), longest=int(lens.max()),
                most_new=int(new.max()), q=_normal(gen, (tokens, case["q_heads"], dim)), pool_k=_normal(gen, (total_pages, hkv, PAGE, dim)))


def _prepare_attend(case, rng, gen):
    st = _paged(case, rng, gen)
    st["pool_v"] = _normal(gen, st["pool_k"].shape)
    shape = st["q"].shape
    if case["prior"]:         # the same rows over a shared prompt, attended before
        st["prior_out"] = (_normal(gen, shape, torch.float32) * 0.05).to(torch.bfloat16)
        st["prior_lse"] = torch.randn(shape[:2], generator=gen, device=DEVICE) * 0.1 + 8.5
    st["out"] = torch.empty(shape, dtype=torch.bfloat16, device=DEVICE)
    st["lse"] = torch.empty(shape[:2], dtype=torch.float32, device=DEVICE)
    return st


def _prepare_weights(case, rng, gen):
    st = _paged(case, rng, gen)
    scores = _scores(st)
    st["lse"] = _from_padded(st, torch.logsumexp(scores, -1))
    del scores
    cells = st["pool_k"].shape[:3]
    st["weights"] = torch.rand(cells, generator=gen, device=DEVICE) ** 8
    st["weights_out"] = torch.zeros(cells, device=DEVICE)
    return st


def _prepare_evict(case, rng, gen):
    n = case["samples"]
    lens = _lengths(rng, n, case["held_lo"], case["held"])
    used = (lens + PAGE - 1) // PAGE
    indptr = _scan(used + rng.integers(0, 3, n))               # lists have room for pages to come
    total_pages = _pool_pages(n, case["held_lo"], case["held"], 0)
    perm = rng.permutation(total_pages)
    indices = np.full(n * (case["held"] // PAGE + 3), -1, np.int64)
    sample = np.repeat(np.arange(n), used)
    at = np.arange(len(sample)) - np.repeat(_scan(used)[:-1], used)
    indices[indptr[sample] + at] = perm[:len(sample)]
    free = np.full(total_pages, -1, np.int64)
    free[:total_pages - len(sample)] = perm[len(sample):]
    return dict(case=case, kv_lens=_i32(lens), page_indptr=_i32(indptr), page_indices=_i32(indices), budgets=_i32(np.full(n, case["budget"])),
                free_pages=_i32(free), free_count=_i32([total_pages - len(sample)]),
                weights=torch.rand((total_pages, case["kv_heads"], PAGE), generator=gen, device=DEVICE) ** 8,
                indices_out=torch.empty(len(indices), dtype=torch.int32, device=DEVICE), lens_out=torch.empty(n, dtype=torch.int32, device=DEVICE),
                count_out=torch.empty(1, dtype=torch.int32, device=DEVICE))


def _prepare_logprobs(case, rng, gen):
    rows, vocab = case["rows"], case["vocab"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    logits = torch.zeros((rows, (vocab + 7) // 8 * 8), dtype=dtype, device=DEVICE)[:, :vocab]
    logits.copy_(torch.randn((rows, vocab), generator=gen, device=DEVICE) * 2.5)
    # a grammar lets one row in four have a tenth of the vocabulary
    masked = torch.from_numpy(rng.random(rows) < 0.25).to(DEVICE).view(-1, 1)
    logits.masked_fill_(masked & (torch.rand((rows, vocab), generator=gen, device=DEVICE) < 0.9), -math.inf)
    f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=DEVICE)  # noqa: E731
    return dict(case=case, logits=logits, tokens=_i32(rng.integers(0, vocab, rows)),
                temperature=torch.from_numpy(rng.choice([0.4, 0.7, 1.0], rows).astype(np.float32)).to(DEVICE), logprobs=f32(rows), entropy=f32(rows),
                top_ids=torch.empty((rows, case["top"]), dtype=torch.int32, device=DEVICE), top_logprobs=f32(rows, case["top"]))


# -------------------------------------------------------------------------------------------------------------- runs
def run(state):
    op = state["case"]["op"]
    if own:
        return {"store": _own_store, "attend": _own_attend, "weights": _own_weights, "evict": _own_evict, "logprobs": _own_logprobs}[op](state)
    return {"store": _plain_store, "attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict, "logprobs": _plain_logprobs}[op](state)


def _own_store(st):
    from paper_2502_02534_b200 import store_kv
    store_kv(st["k"], st["v"], st["slots"], st["pool_k"], st["pool_v"])
    return {"k": st["pool_k"], "v": st["pool_v"]}


def _own_attend(st):
    from paper_2502_02534_b200 import attend_paged
    attend_paged(st["q"], st["pool_k"], st["pool_v"], st["page_indptr"], st["page_indices"], st["kv_lens"], st["q_indptr"], st["out"], st["lse"],
                 prior_out=st.get("prior_out"), prior_lse=st.get("prior_lse"))
    return {"out": st["out"], "lse": st["lse"]}


def _own_weights(st):
    from paper_2502_02534_b200 import accumulate_weights
    accumulate_weights(st["q"], st["lse"], st["pool_k"], st["page_indptr"], st["page_indices"], st["kv_lens"], st["q_indptr"], st["weights"],
                       weights_out=st["weights_out"])
    return {"weights": st["weights_out"]}


def _own_evict(st):
    from paper_2502_02534_b200 import evict_pages
    evict_pages(st["weights"], st["page_indptr"], st["page_indices"], st["kv_lens"], st["budgets"], st["case"]["recent"], st["free_pages"],
                st["free_count"], page_indices_out=st["indices_out"], lens_out=st["lens_out"], free_count_out=st["count_out"])
    return {k: st[k] for k in ("indices_out", "lens_out", "free_pages", "count_out")}


def _own_logprobs(st):
    from paper_2502_02534_b200 import token_logprobs
    token_logprobs(st["logits"], st["tokens"], st["case"]["top"], temperature=st["temperature"], logprobs=st["logprobs"], entropy=st["entropy"],
                   top_ids=st["top_ids"], top_logprobs=st["top_logprobs"])
    return {k: st[k] for k in ("logprobs", "entropy", "top_ids", "top_logprobs")}


def _plain_store(st):
    keep = st["slots"] >= 0
    page = torch.where(keep, st["slots"] // PAGE, torch.full_like(st["slots"], st["pool_k"].shape[0]))       # one page more takes the empty rows
    pos = torch.where(keep, st["slots"] % PAGE, torch.zeros_like(st["slots"]))
    pools = torch.cat([torch.stack([st["pool_k"], st["pool_v"]]), torch.zeros_like(st["pool_k"][:1]).expand(2, 1, -1, -1, -1)], 1)
    pools[:, page, :, pos] = torch.stack([st["k"], st["v"]], 1)
    return {"k": pools[0, :-1], "v": pools[1, :-1]}


def _rows(st):
    """Where the padded form [samples, most_new] finds its rows, and which of them exist."""
    first = st["q_indptr"].long()
    at = first[:-1, None] + torch.arange(st["most_new"], device=DEVICE)
    live = at < first[1:, None]
    return torch.clamp(at, max=st["q"].shape[0] - 1), live


def _from_padded(st, x):
    """[samples, kv_heads, most_new, group, ...] -> [tokens, q_heads, ...]"""
    at, live = _rows(st)
    x = x.permute(0, 2, 1, 3, *range(4, x.dim())).flatten(2, 3)
    got = torch.zeros((st["q"].shape[0] + 1, *x.shape[2:]), dtype=x.dtype, device=DEVICE)
    got[torch.where(live, at, torch.full_like(at, st["q"].shape[0]))] = x
    return got[:-1]


def _gathered(st, pool):
    """The sample's keys or values in order, fp32: [samples, kv_heads, keys, dim]."""
    width = (st["longest"] + PAGE - 1) // PAGE
    at = st["page_indptr"][:-1].long().unsqueeze(1) + torch.arange(width, device=DEVICE)
    at = torch.clamp(at, max=st["page_indices"].numel() - 1)
    x = pool[st["page_indices"][at].long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], width * PAGE, -1).float()


def _scores(st):
    """Scaled scores, -inf where a row does not see a key: [samples, kv_heads, most_new, group, keys], fp32."""
    case = st["case"]
    hkv, g, dim = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"]
    at, live = _rows(st)
    q = st["q"][at].float().unflatten(2, (hkv, g)).permute(0, 2, 1, 3, 4) * dim ** -0.5     # [samples, hkv, most_new, g, dim]
    k = _gathered(st, st["pool_k"])
    s = torch.matmul(q.flatten(2, 3), k.transpose(-1, -2)).unflatten(2, (-1, g))
    new = st["q_indptr"][1:] - st["q_indptr"][:-1]
    sees = (st["kv_lens"] - new)[:, None] + torch.arange(st["most_new"], device=DEVICE)      # last key of each row
    seen = (torch.arange(s.shape[-1], device=DEVICE) <= sees.unsqueeze(-1)) & live.unsqueeze(-1)
    return s.masked_fill_(~seen[:, None, :, None], -math.inf)


def _plain_attend(st):
    s = _scores(st)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = _from_padded(st, (top + torch.log(total)).squeeze(-1))
    out = torch.matmul(p.flatten(2, 3), _gathered(st, st["pool_v"])).unflatten(2, (st["most_new"], -1))
    out = _from_padded(st, out / torch.where(total > 0, total, torch.ones_like(total)))
    if "prior_out" in st:
        both = torch.logaddexp(lse, st["prior_lse"])
        out = out * torch.exp(lse - both).unsqueeze(-1) + st["prior_out"].float() * torch.exp(st["prior_lse"] - both).unsqueeze(-1)
        lse = both
    return {"out": out.to(torch.bfloat16), "lse": lse}


def _plain_weights(st):
    case = st["case"]
    s = _scores(st)
    at, live = _rows(st)
    lse = st["lse"][at].unflatten(2, (case["kv_heads"], -1)).permute(0, 2, 1, 3).unsqueeze(-1)
    got = s.sub_(lse).masked_fill_(~live[:, None, :, None, None], -math.inf).exp_().sum((2, 3))             # [samples, kv_heads, keys]
    width = got.shape[-1] // PAGE
    pages = (st["kv_lens"].long() + PAGE - 1) // PAGE
    entry = torch.arange(width, device=DEVICE)
    spare = st["weights"].shape[0]
    page = st["page_indices"][torch.clamp(st["page_indptr"][:-1].long().unsqueeze(1) + entry, max=st["page_indices"].numel() - 1)].long()
    page = torch.where(entry < pages.unsqueeze(1), page, torch.full_like(page, spare))
    new = (st["q_indptr"][1:] - st["q_indptr"][:-1]).view(-1, 1, 1)
    key = torch.arange(width * PAGE, device=DEVICE)
    before = torch.cat([st["weights"], torch.zeros_like(st["weights"][:1])])[page].transpose(1, 2).flatten(2)     # [samples, kv_heads, keys]
    lens = st["kv_lens"].view(-1, 1, 1)
    got = torch.where(key < lens - new, before + got, got)                                                      # new tokens start from nothing
    out = torch.cat([st["weights_out"], torch.zeros_like(st["weights_out"][:1])])
    cells = torch.where((key < lens).expand_as(got), got, torch.zeros_like(got))
    out[page] = cells.unflatten(2, (width, PAGE)).transpose(1, 2)
    return {"weights": out[:-1]}


def _plain_evict(st):
    n = st["kv_lens"].numel()
    recent = st["case"]["recent"]
    lens = st["kv_lens"].long()
    pages = (lens + PAGE - 1) // PAGE
    budget = st["budgets"].long()
    width = st["case"]["held"] // PAGE + 1
    entry = torch.arange(width, device=DEVICE)
    at = st["page_indptr"][:-1].long().unsqueeze(1) + entry
    page = st["page_indices"][at].long()
    held = entry < pages.unsqueeze(1)
    weight = st["weights"].flatten(1).amax(1)[torch.clamp(page, min=0)]
    newest = (entry >= (pages - torch.clamp(budget, max=recent)).unsqueeze(1)) & held
    weight = torch.where(newest, torch.full_like(weight, math.inf), torch.where(held, weight, torch.full_like(weight, -math.inf)))
    order = torch.sort(weight, dim=1, descending=True, stable=True).indices                # of equal weights the older page stays
    rank = torch.empty_like(order).scatter_(1, order, entry.expand(n, -1))
    stays = held & (rank < budget.unsqueeze(1))
    goes = held & ~stays
    out = torch.cat([st["page_indices"], st["page_indices"][:1]])                          # one entry more takes what has no place
    spare = out.numel() - 1
    out[torch.where(held, at, torch.full_like(at, spare))] = -1
    to = st["page_indptr"][:-1].long().unsqueeze(1) + torch.cumsum(stays, 1) - 1
    out[torch.where(stays, to, torch.full_like(to, spare))] = page.int()
    gone = torch.cumsum(goes.flatten(), 0).view(n, -1)
    free = torch.cat([st["free_pages"], st["free_pages"][:1]])
    count = st["free_count"].long()
    free[torch.where(goes, count + gone - 1, torch.full_like(gone, free.numel() - 1))] = page.int()
    return {"indices_out": out[:-1], "lens_out": (lens - PAGE * goes.sum(1)).int(), "free_pages": free[:-1], "count_out": (count + gone[-1, -1]).int()}


def _plain_logprobs(st):
    top = st["case"]["top"]
    x = st["logits"].float() / st["temperature"].unsqueeze(1)
    most = x.amax(1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(1, keepdim=True)
    norm = most + torch.log(total)
    logp = x - norm
    entropy = -torch.where(e > 0, e / total * logp, torch.zeros_like(e)).sum(1)
    index = torch.sort(st["logits"].float(), dim=1, descending=True, stable=True).indices[:, :top]           # of equal logits the lower token
    return {"logprobs": logp.gather(1, st["tokens"].long().unsqueeze(1)).squeeze(1), "entropy": entropy, "top_ids": index.int(),
            "top_logprobs": logp.gather(1, index)}


# -------------------------------------------------------------------------------------------------------------- work
def _means(case):
    """Mean over the seeds of: new tokens, cached and new tokens, scores per query head."""
    new = _new_lens(case).astype(np.float64)
    cached = (case["cached_lo"] + case["cached"]) / 2
    return new.sum(), case["samples"] * cached + new.sum(), (new * cached + new * (new + 1) / 2).sum()


def work(case):
    op = case["op"]
    if op == "store":
        tokens = float(_new_lens(case).sum())
        return {"bytes": tokens * (8.0 * case["kv_heads"] * case["dim"] + 8), "flops": 0}
    if op in ("attend", "weights"):
        rows, keys, scores = _means(case)
        row, qrow = case["kv_heads"] * case["dim"], case["q_heads"] * case["dim"]
        if op == "attend":
            moved = 4.0 * keys * row + rows * (4.0 * qrow + 4 * case["q_heads"]) * (1.5 if case["prior"] else 1)
            return {"bytes": moved + keys / 4, "flops": 4.0 * scores * qrow}
        return {"bytes": 2.0 * keys * row + 8.0 * keys * case["kv_heads"] + rows * (2.0 * qrow + 4 * case["q_heads"]) + keys / 4,
                "flops": 2.0 * scores * qrow}
    if op == "evict":
        pages = case["samples"] * (case["held_lo"] + case["held"]) / 2 / PAGE
        return {"bytes": pages * (4.0 * PAGE * case["kv_heads"] + 12), "flops": pages * PAGE * case["kv_heads"]}
    size = 2 if case["dtype"] == "bf16" else 4
    return {"bytes": float(size) * case["rows"] * case["vocab"] + case["rows"] * (16 + 8 * case["top"]), "flops": 6.0 * case["rows"] * case["vocab"]}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    if case["op"] in ("store", "evict"):
        return None            # moved values and whole numbers: nothing is computed
    st = prepare(case, seed)
    return {"attend": _exact_attend, "weights": _exact_weights, "logprobs": _exact_logprobs}[case["op"]](st)


def _each(st):
    """Of every (sample, KV head): its rows, its pages and its scores [rows, group, keys] in 64 bits, unseen keys at -inf."""
    case = st["case"]
    g, dim = case["q_heads"] // case["kv_heads"], case["dim"]
    rows, lists, lens, ids = st["q_indptr"].tolist(), st["page_indptr"].tolist(), st["kv_lens"].tolist(), st["page_indices"].long()
    for s in range(case["samples"]):
        a, b, length = rows[s], rows[s + 1], lens[s]
        mine = ids[lists[s]:lists[s] + -(-length // PAGE)]
        hidden = torch.ones((b - a, length), dtype=torch.bool, device=DEVICE).triu(length - (b - a) + 1).unsqueeze(1)
        for h in range(case["kv_heads"]):
            k = st["pool_k"][mine, h].reshape(-1, dim)[:length].double()
            x = st["q"][a:b, h * g:(h + 1) * g].double()
            yield s, h, slice(a, b), slice(h * g, (h + 1) * g), mine, length, (x @ k.T / math.sqrt(dim)).masked_fill(hidden, -math.inf)


def _exact_attend(st):
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(st["q"].shape[:2], dtype=torch.float64, device=DEVICE)
    for s, h, rows, heads, mine, length, x in _each(st):
        v = st["pool_v"][mine, h].reshape(-1, st["case"]["dim"])[:length].double()
        lse[rows, heads] = torch.logsumexp(x, 2)
        out[rows, heads] = torch.softmax(x, 2) @ v
    if st["case"]["prior"]:
        a = torch.sigmoid(lse - st["prior_lse"].double()).unsqueeze(2)          # share of the cache
        out = a * out + (1 - a) * st["prior_out"].double()
        lse = torch.logsumexp(torch.stack([lse, st["prior_lse"].double()]), 0)
    return {"out": out, "lse": lse}


def _exact_weights(st):
    got = st["weights_out"].double()
    new = (st["q_indptr"][1:] - st["q_indptr"][:-1]).tolist()
    for s, h, rows, heads, mine, length, x in _each(st):
        w = torch.exp(x - st["lse"][rows, heads].double().unsqueeze(2)).sum((0, 1))
        old = st["weights"][mine, h].reshape(-1)[:length].double()
        old[length - new[s]:] = 0
        cells = torch.zeros(len(mine) * PAGE, dtype=torch.float64, device=DEVICE)
        cells[:length] = old + w
        got[mine, h] = cells.view(-1, PAGE)
    return {"weights": got}


def _exact_logprobs(st):
    x = st["logits"].double() / st["temperature"].double().unsqueeze(1)
    p = torch.softmax(x, 1)
    logp = torch.log_softmax(x, 1)
    entropy = -torch.special.xlogy(p, p).sum(1)
    rows = torch.arange(x.shape[0], device=DEVICE)
    index = torch.sort(st["logits"].double(), dim=1, descending=True, stable=True).indices[:, :st["case"]["top"]]
    return {"logprobs": logp[rows, st["tokens"].long()], "entropy": entropy, "top_ids": index.int(), "top_logprobs": logp.gather(1, index)}
