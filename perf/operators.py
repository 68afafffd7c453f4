"""Cases that measure the operators around a decode step: page tables built on the GPU, the 4-bit K/V cache (written, read
back and attended over) and the rules applied to logits before a token is drawn.

``own`` chooses between the plain form (elementary torch operations, this file) and the library's entry points.  Both take
what ``prepare`` makes.  Shapes follow the configurations of ``psa_workloads`` (8 to 256 samples, 8 KV heads of 64 or 128
channels, generated answers of up to 4096 tokens, shared prompts of up to 32768) and the 131072-token vocabulary of the
sampling tests.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16          # tokens per page
DEVICE = "cuda"
GROUP = 32         # channels that share a scale and an offset in the 4-bit cache


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a running batch: a slot for one new token of every sample
        dict(name="pages-step", op="pages", mode="extend", samples=256, held=4096, new_lo=1, new=1),
        # samples resumed with answers of different lengths: whole page lists and the slot of every token
        dict(name="pages-admit", op="pages", mode="build", samples=2048, held=0, new_lo=0, new=4096),
        # the K/V of one new token per sample into the 4-bit cache, and back
        dict(name="kv4-step", op="kv4", samples=32, new_lo=1, new=1, kv_heads=8, dim=128),
        # answers of many lengths moved into the cache at once, and read back to become a shared prompt
        dict(name="kv4-answers", op="kv4", samples=64, new_lo=0, new=2048, kv_heads=8, dim=128),
        # the smallest configuration: 8 samples of one short prompt, 64 channels
        dict(name="decode-small", op="decode", prompts=1, samples=8, prefix_lo=512, prefix=512, suffix_lo=1, suffix=128,
             q_heads=8, kv_heads=2, dim=64),
        # the cache alone, no shared prompt, one query head per KV head
        dict(name="decode-own", op="decode", prompts=1, samples=64, prefix_lo=0, prefix=0, suffix_lo=1, suffix=4096,
             q_heads=8, kv_heads=8, dim=128),
        # 32 samples of one prompt
        dict(name="decode-mid", op="decode", prompts=1, samples=32, prefix_lo=4096, prefix=4096, suffix_lo=0, suffix=1024,
             q_heads=32, kv_heads=8, dim=128),
        # 256 samples of one prompt, answers of up to 4096 tokens: the library's headline batch
        dict(name="decode-large", op="decode", prompts=1, samples=256, prefix_lo=8192, prefix=8192, suffix_lo=0, suffix=4096,
             q_heads=64, kv_heads=8, dim=128),
        # a few answers with a small vocabulary
        dict(name="rules-few", op="rules", rows=8, vocab=3001, history=128, biases=16, dtype="f32"),
        # a full batch over a large vocabulary
        dict(name="rules-batch", op="rules", rows=256, vocab=131072, history=1024, biases=64, dtype="bf16"),
        # which tokens one short prompt holds
        dict(name="mark-one", op="mark", rows=1, ids=512, vocab=3001),
        # which tokens each of 64 long prompts holds
        dict(name="mark-many", op="mark", rows=64, ids=32768, vocab=131072),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["pages", "kv4", "decode", "decode", "rules", "mark"])
    if op == "pages":
        mode = rng.choice(["extend", "build"])
        samples = _log_int(rng, 1, 2048)
        return dict(op=op, mode=mode, samples=samples, held=_log_int(rng, 1, 4096) if mode == "extend" else 0,
                    new_lo=rng.choice([0, 1]), new=_log_int(rng, 1, 4096))
    if op == "kv4":
        return dict(op=op, samples=_log_int(rng, 1, 64), new_lo=rng.choice([0, 1]), new=_log_int(rng, 1, 2048),
                    kv_heads=rng.choice([1, 2, 8]), dim=rng.choice([64, 128]))
    if op == "decode":
        prompts = rng.choice([1, 1, 2, 5])
        samples = _log_int(rng, 1, 256 // prompts)
        kv = rng.choice([1, 2, 8])
        prefix = rng.choice([0, _log_int(rng, 1, 8192)])
        return dict(op=op, prompts=prompts, samples=samples, prefix_lo=prefix // 2, prefix=prefix, suffix_lo=rng.choice([0, 1]),
                    suffix=_log_int(rng, 1, 4096), q_heads=kv * rng.choice([1, 2, 4, 8]), kv_heads=kv, dim=rng.choice([64, 128]))
    if op == "rules":
        return dict(op=op, rows=_log_int(rng, 1, 256), vocab=_log_int(rng, 100, 131072), history=_log_int(rng, 1, 1024),
                    biases=_log_int(rng, 1, 64), dtype=rng.choice(["bf16", "f32"]) if rng.random() < 0.5 else "bf16")
    return dict(op=op, rows=_log_int(rng, 1, 64), ids=_log_int(rng, 1, 32768), vocab=_log_int(rng, 100, 131072))


# ------------------------------------------------------------------------------------------------------------ inputs
def _lengths(rng, n, lo, hi):
    """n whole numbers spread evenly over [lo, hi], in random order."""
    at = (np.arange(n) + rng.random(n)) / n
    return rng.permutation(np.minimum(hi, lo + np.floor((hi - lo + 1) * at))).astype(np.int32)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)


def _normal(gen, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(dtype)


def _quantise(x):
    """x [..., D] -> (codes [..., D] 0..15, scale and offset [..., D / 32], fp32 values of bf16 numbers)."""
    g = x.float().unflatten(-1, (-1, GROUP))
    low, high = g.amin(-1), g.amax(-1)
    scale = ((high - low) / 15).to(torch.bfloat16).float()
    codes = torch.round((g - low.unsqueeze(-1)) / scale.unsqueeze(-1))
    codes = torch.where(scale.unsqueeze(-1) > 0, codes, torch.zeros_like(codes)).clamp(0, 15)
    return codes.flatten(-2), scale, low


def _swizzle(dim):
    """Place of chunk (token, group) of a page's codes, in 16-byte chunks: [16, dim / 32]."""
    groups = dim // GROUP
    t = torch.arange(PAGE, device=DEVICE).view(-1, 1)
    g = torch.arange(groups, device=DEVICE).view(1, -1)
    return t * groups + (g ^ ((t >> 1) & 3 if dim == 128 else (t >> 2) & 1))


def _pack(k, v):
    """k, v [pages, heads, 16, D] bf16 -> cells [pages, heads, 20 D] uint8 (the layout include/psa.h describes)."""
    dim = k.shape[-1]
    lead = k.shape[:2]
    parts, params = [], []
    place = _swizzle(dim).flatten()
    for x in (k, v):
        codes, scale, low = _quantise(x)
        codes = codes.to(torch.uint8)
        chunks = (codes[..., 0::2] | (codes[..., 1::2] << 4)).view(*lead, PAGE * dim // GROUP, 16)
        out = torch.empty_like(chunks)
        out[:, :, place] = chunks
        parts.append(out.flatten(2))
        params.append(torch.cat([scale, low], -1).to(torch.bfloat16))
    if dim == 128:
        parts += [p.contiguous().view(torch.uint8).flatten(2) for p in params]
    else:
        parts.append(torch.cat(params, -1).contiguous().view(torch.uint8).flatten(2))
    return torch.cat(parts, -1)


def _prefix_lengths(case):
    """Prompt lengths, the same for every seed: they shape the plan."""
    return _lengths(np.random.default_rng(9), case["prompts"], case["prefix_lo"], case["prefix"])


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    return {"pages": _prepare_pages, "kv4": _prepare_kv4, "decode": _prepare_decode, "rules": _prepare_rules,
            "mark": _prepare_mark}[case["op"]](case, rng, gen)


def _most_entries(case):
    """List entries a sample has at most: its longest answer and 63 tokens more."""
    return (case["held"] + case["new"] + 63 + PAGE - 1) // PAGE


def _prepare_pages(case, rng, gen):
    n = case["samples"]
    held = _lengths(rng, n, 0, case["held"]) if case["held"] else np.zeros(n, np.int32)
    new = _lengths(rng, n, case["new_lo"], case["new"])
    reserve = held + new + rng.integers(0, 64, n).astype(np.int32)
    slots = (reserve + PAGE - 1) // PAGE
    indptr = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    total = int(indptr[-1])
    perm = rng.permutation(total + 32).astype(np.int32)
    indices = np.full(n * _most_entries(case), -1, np.int32)
    used = 0
    for s in range(n if case["held"] else 0):
        k = (int(held[s]) + PAGE - 1) // PAGE
        indices[indptr[s]:indptr[s] + k] = perm[used:used + k]
        used += k
    st = dict(case=case, held=_i32(held), new=_i32(new), reserve=_i32(reserve), page_indptr=_i32(indptr), page_indices=_i32(indices),
              free_pages=_i32(perm[used:]), free_count=_i32([len(perm) - used]), max_tokens=n * case["new"])
    st.update(lens_out=torch.empty(n, dtype=torch.int32, device=DEVICE), count_out=torch.empty(1, dtype=torch.int32, device=DEVICE),
              token_indptr=torch.empty(n + 1, dtype=torch.int32, device=DEVICE),
              slot_map=torch.empty(max(1, st["max_tokens"]), dtype=torch.int64, device=DEVICE))
    if own:
        from paper_2502_02534_b200 import page_table_scratch
        st["scratch"] = page_table_scratch(n)
    return st


def _slots(rng, new, total_pages):
    """A slot for every token of every sample: its pages scattered over the pool, as a running server leaves them."""
    pages = (new.astype(np.int64) + PAGE - 1) // PAGE
    ids = rng.permutation(total_pages)[:int(pages.sum())]
    first = np.concatenate([[0], np.cumsum(pages)])[:-1]
    sample = np.repeat(np.arange(len(new)), new)
    pos = np.arange(len(sample)) - np.repeat(np.concatenate([[0], np.cumsum(new.astype(np.int64))])[:-1], new)
    return ids[first[sample] + pos // PAGE] * PAGE + pos % PAGE


def _prepare_kv4(case, rng, gen):
    new = _lengths(np.random.default_rng(9), case["samples"], case["new_lo"], case["new"])      # the same for every seed
    heads, dim = case["kv_heads"], case["dim"]
    total_pages = int(((new.astype(np.int64) + PAGE - 1) // PAGE).sum()) + 8
    slots = _slots(rng, new, total_pages)
    slots = np.concatenate([slots, np.full(3, -1)])           # a batch padded to its captured size ends in empty rows
    tokens = len(slots)
    return dict(case=case, slots=torch.from_numpy(slots.astype(np.int64)).to(DEVICE), k=_normal(gen, (tokens, heads, dim)),
                v=_normal(gen, (tokens, heads, dim)),
                pool=torch.zeros((total_pages, heads, 20 * dim), dtype=torch.uint8, device=DEVICE),
                out_k=torch.zeros((tokens, heads, dim), dtype=torch.bfloat16, device=DEVICE),
                out_v=torch.zeros((tokens, heads, dim), dtype=torch.bfloat16, device=DEVICE))


def _prepare_decode(case, rng, gen):
    n = case["prompts"] * case["samples"]
    hq, hkv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    prefix = _prefix_lengths(case)
    suffix = _lengths(rng, n, case["suffix_lo"], case["suffix"])
    pages = (suffix + PAGE - 1) // PAGE
    indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    total_pages = int(indptr[-1]) + int(indptr[-1]) // 8 + 1
    indices = rng.permutation(total_pages)[:int(indptr[-1])].astype(np.int32)
    pool = torch.empty((total_pages, hkv, 20 * dim), dtype=torch.uint8, device=DEVICE)
    for a in range(0, total_pages, 4096):
        b = min(total_pages, a + 4096)
        pool[a:b] = _pack(_normal(gen, (b - a, hkv, PAGE, dim)), _normal(gen, (b - a, hkv, PAGE, dim)))
    tokens = int(prefix.sum())
    st = dict(case=case, prefix_lens=_i32(prefix), suffix_lens=_i32(suffix), page_indptr=_i32(indptr),
              page_indices=_i32(indices if len(indices) else np.zeros(1)), pool=pool, longest=int(suffix.max()),
              q=_normal(gen, (n, hq, dim)), prefix_k=_normal(gen, (tokens, hkv, dim)), prefix_v=_normal(gen, (tokens, hkv, dim)),
              out=torch.empty((n, hq, dim), dtype=torch.bfloat16, device=DEVICE),
              lse=torch.empty((n, hq), dtype=torch.float32, device=DEVICE))
    if own:
        from paper_2502_02534_b200 import Plan
        st["plan"] = Plan(prefix, np.full(case["prompts"], case["samples"], np.int32), suffix, num_q_heads=hq, num_kv_heads=hkv,
                          head_dim=dim, sm_scale=dim ** -0.5, out_dtype="bf16")
        st["plan"].bind_workspace()
    return st


def _prepare_rules(case, rng, gen):
    rows, vocab, words = case["rows"], case["vocab"], (case["vocab"] + 31) // 32
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    stride = (vocab + 7) // 8 * 8
    buf = lambda: torch.zeros((rows, stride), dtype=dtype, device=DEVICE)[:, :vocab]  # noqa: E731
    logits = buf()
    logits.copy_(torch.randn((rows, vocab), generator=gen, device=DEVICE) * 2.5)
    # generated tokens repeat themselves: few ids make up most of an answer
    history = np.minimum(vocab - 1, np.floor(vocab * rng.random((rows, case["history"])) ** 3)).astype(np.int32)
    prompts = max(1, rows // 64)
    prompt_bits = rng.integers(0, 2 ** 32, (prompts, words), dtype=np.uint64) & rng.integers(0, 2 ** 32, (prompts, words), dtype=np.uint64) \
        & rng.integers(0, 2 ** 32, (prompts, words), dtype=np.uint64) & rng.integers(0, 2 ** 32, (prompts, words), dtype=np.uint64)
    # one grammar state lets few tokens through, the other all but a few; some rows have none
    allow = rng.integers(0, 2 ** 32, (2, words), dtype=np.uint64)
    allow[0] &= rng.integers(0, 2 ** 32, words, dtype=np.uint64) & rng.integers(0, 2 ** 32, words, dtype=np.uint64)
    allow[1] |= rng.integers(0, 2 ** 32, words, dtype=np.uint64) | rng.integers(0, 2 ** 32, words, dtype=np.uint64)
    count = _lengths(rng, rows, 0, case["biases"])
    indptr = np.concatenate([[0], np.cumsum(count)]).astype(np.int32)
    bits = lambda a: torch.from_numpy(a.astype(np.uint32).view(np.int32)).to(DEVICE)  # noqa: E731
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(DEVICE)  # noqa: E731
    return dict(case=case, logits=logits, out=buf(), history=_i32(history), history_lens=_i32(_lengths(rng, rows, 0, case["history"])),
                repetition=f32(rng.choice([1.0, 1.1, 1.3], rows)), frequency=f32(rng.choice([0.0, 0.2, 0.5], rows)),
                presence=f32(rng.choice([0.0, 0.4], rows)), prompt_bits=bits(prompt_bits), prompt_rows=_i32(np.arange(rows) % prompts),
                mask_bits=bits(allow), mask_rows=_i32(rng.choice([-1, 0, 1], rows)), bias_indptr=_i32(indptr),
                bias_ids=_i32(rng.integers(0, vocab, int(indptr[-1]) + 1)), bias_values=f32(rng.normal(0, 3, int(indptr[-1]) + 1)))


def _prepare_mark(case, rng, gen):
    lens = _lengths(rng, case["rows"], case["ids"] // 2, case["ids"])
    indptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    ids = np.minimum(case["vocab"] - 1, np.floor(case["vocab"] * rng.random(int(indptr[-1]) + 1) ** 2))
    return dict(case=case, ids=_i32(ids), indptr=_i32(indptr),
                bits=torch.empty((case["rows"], (case["vocab"] + 31) // 32), dtype=torch.int32, device=DEVICE))


# -------------------------------------------------------------------------------------------------------------- runs
def run(state):
    op = state["case"]["op"]
    if own:
        return {"pages": _own_pages, "kv4": _own_kv4, "decode": _own_decode, "rules": _own_rules, "mark": _own_mark}[op](state)
    return {"pages": _plain_pages, "kv4": _plain_kv4, "decode": _plain_decode, "rules": _plain_rules, "mark": _plain_mark}[op](state)


def _own_pages(st):
    from paper_2502_02534_b200 import build_page_table, extend_page_table
    if st["case"]["mode"] == "build":
        build_page_table(st["new"], st["free_pages"], st["free_count"], st["page_indptr"], st["page_indices"], st["token_indptr"],
                         st["slot_map"], reserve_lens=st["reserve"], lens_out=st["lens_out"], free_count_out=st["count_out"],
                         scratch=st["scratch"])
    else:
        extend_page_table(st["held"], st["new"], st["free_pages"], st["free_count"], st["page_indptr"], st["page_indices"],
                          st["token_indptr"], st["slot_map"], max_lens=st["reserve"], lens_out=st["lens_out"],
                          free_count_out=st["count_out"], scratch=st["scratch"])
    return {k: st[k] for k in ("page_indptr", "page_indices", "token_indptr", "slot_map", "lens_out", "count_out")}


def _own_kv4(st):
    from paper_2502_02534_b200 import load_kv4, store_kv4
    store_kv4(st["k"], st["v"], st["slots"], st["pool"])
    load_kv4(st["pool"], st["slots"], st["out_k"], st["out_v"])
    return {"k": st["out_k"], "v": st["out_v"]}


def _own_decode(st):
    from paper_2502_02534_b200 import decode_kv4
    decode_kv4(st["plan"], st["q"], st["prefix_k"], st["prefix_v"], st["pool"], st["page_indptr"], st["page_indices"],
               st["suffix_lens"], st["out"], st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_rules(st):
    from paper_2502_02534_b200 import process_logits
    process_logits(st["logits"], st["out"], repetition=st["repetition"], frequency=st["frequency"], presence=st["presence"],
                   history=st["history"], history_lens=st["history_lens"], prompt_bits=st["prompt_bits"], prompt_rows=st["prompt_rows"],
                   bias_indptr=st["bias_indptr"], bias_ids=st["bias_ids"], bias_values=st["bias_values"],
                   mask_bits=st["mask_bits"], mask_rows=st["mask_rows"])
    return {"logits": st["out"]}


def _own_mark(st):
    from paper_2502_02534_b200 import mark_tokens
    mark_tokens(st["ids"], st["indptr"], st["case"]["vocab"], st["bits"])
    return {"bits": st["bits"]}


def _scan0(x):
    """[0, x0, x0 + x1, ...] as int64."""
    return torch.cat([torch.zeros(1, dtype=torch.int64, device=x.device), torch.cumsum(x.to(torch.int64), 0)])


def _plain_pages(st):
    build = st["case"]["mode"] == "build"
    held, new = st["held"].long(), st["new"].long()
    n = held.numel()
    if build:
        indptr = _scan0((st["reserve"].long() + PAGE - 1) // PAGE)
        indices = torch.full_like(st["page_indices"], -1)
    else:
        indptr = st["page_indptr"].long()
        indices = st["page_indices"].clone()
    first_new = (held + PAGE - 1) // PAGE                       # first list entry without a page
    last = (held + new + PAGE - 1) // PAGE
    need = torch.clamp(last - first_new, min=0)
    base = _scan0(need)
    count = st["free_count"].long()
    # every list entry that gets a page in this call
    entry = torch.arange(indices.numel(), device=DEVICE)
    s = torch.clamp(torch.searchsorted(indptr, entry, right=True) - 1, 0, n - 1)
    j = entry - indptr[s]
    gets = (entry < indptr[-1]) & (j >= first_new[s]) & (j < last[s])
    top = torch.clamp(count - 1 - (base[s] + j - first_new[s]), min=0).clamp(max=st["free_pages"].numel() - 1)
    indices = torch.where(gets, st["free_pages"][top], indices)
    # the slot of every new token
    tokens = _scan0(new)
    t = torch.arange(st["max_tokens"], device=DEVICE)
    s = torch.clamp(torch.searchsorted(tokens, t, right=True) - 1, 0, n - 1)
    pos = held[s] + t - tokens[s]
    entry = torch.clamp(indptr[s] + pos // PAGE, 0, indices.numel() - 1)
    slot = indices[entry].long() * PAGE + pos % PAGE
    slot = torch.where(t < tokens[-1], slot, torch.full_like(slot, -1))
    if not st["max_tokens"]:
        slot = torch.full_like(st["slot_map"], -1)
    return {"page_indptr": indptr.int(), "page_indices": indices, "token_indptr": tokens.int(), "slot_map": slot,
            "lens_out": (held + new).int(), "count_out": (count - base[-1]).int()}


def _plain_kv4(st):
    keep = (st["slots"] >= 0).view(-1, 1, 1)
    got = {}
    for name in ("k", "v"):
        codes, scale, low = _quantise(st[name])
        value = codes.unflatten(-1, (-1, GROUP)) * scale.unsqueeze(-1) + low.unsqueeze(-1)
        got[name] = torch.where(keep, value.flatten(-2), torch.zeros_like(codes)).to(torch.bfloat16)
    return got


def _unpack(cells, dim):
    """cells [..., 20 D] -> (k, v) [..., 16, D] fp32."""
    lead, half, groups = cells.shape[:-1], PAGE * dim // 2, dim // GROUP
    place = _swizzle(dim).flatten()
    params = cells[..., 2 * half:].contiguous().view(torch.bfloat16).float()
    if dim == 128:
        params = params.view(*lead, 2, PAGE, 2, groups)
    else:
        params = params.view(*lead, PAGE, 2, 2, groups).transpose(-4, -3)
    out = []
    for i in range(2):
        chunks = cells[..., i * half:(i + 1) * half].view(*lead, PAGE * groups, 16)[..., place, :].view(*lead, PAGE, groups, 16)
        codes = torch.stack([chunks & 15, chunks >> 4], -1).flatten(-2).float()
        scale, low = params[..., i, :, 0, :], params[..., i, :, 1, :]
        out.append((codes * scale.unsqueeze(-1) + low.unsqueeze(-1)).flatten(-2))
    return out


def _plain_decode(st):
    case = st["case"]
    hkv, dim, per = case["kv_heads"], case["dim"], case["samples"]
    n = case["prompts"] * per
    g = case["q_heads"] // hkv
    q = st["q"].float().view(n, hkv, g, dim) * dim ** -0.5
    scores, values, shared = [], [], st["prefix_k"].shape[0] > 0
    if not st["longest"] and not shared:
        return {"out": torch.zeros_like(st["q"]), "lse": torch.full((n, hkv * g), -math.inf, device=DEVICE)}
    if st["longest"]:
        width = (st["longest"] + PAGE - 1) // PAGE
        at = torch.clamp(st["page_indptr"][:-1].long().unsqueeze(1) + torch.arange(width, device=DEVICE), max=st["page_indices"].numel() - 1)
        k, v = _unpack(st["pool"][st["page_indices"][at].long()], dim)           # [n, width, hkv, 16, dim]
        k, v = (x.transpose(1, 2).reshape(n, hkv, width * PAGE, dim) for x in (k, v))
        live = torch.arange(width * PAGE, device=DEVICE) < st["suffix_lens"].unsqueeze(1)
        s = torch.matmul(q, k.transpose(-1, -2))
        scores.append(torch.where(live.view(n, 1, 1, -1), s, torch.full_like(s, -math.inf)))
        values.append(torch.where(live.view(n, 1, -1, 1), v, torch.zeros_like(v)))
        del k, v, s
    if shared:
        lens = st["prefix_lens"].long()
        at = _scan0(lens)[:-1].unsqueeze(1) + torch.arange(case["prefix"], device=DEVICE)
        at = torch.clamp(at, max=st["prefix_k"].shape[0] - 1)
        pk, pv = (x[at].float().permute(0, 2, 1, 3) for x in (st["prefix_k"], st["prefix_v"]))      # [prompts, hkv, tokens, dim]
        live = (torch.arange(case["prefix"], device=DEVICE) < lens.unsqueeze(1)).view(-1, 1, 1, case["prefix"])
        qp = q.view(-1, per, hkv, g, dim).permute(0, 2, 1, 3, 4).reshape(-1, hkv, per * g, dim)
        s = torch.matmul(qp, pk.transpose(-1, -2))
        s = torch.where(live, s, torch.full_like(s, -math.inf))
        scores.append(s.view(-1, hkv, per, g, case["prefix"]).permute(0, 2, 1, 3, 4).reshape(n, hkv, g, -1))
        del s
    top = torch.stack([s.amax(-1) for s in scores]).amax(0)
    safe = torch.where(torch.isinf(top), torch.zeros_like(top), top).unsqueeze(-1)
    scores = [torch.exp(s - safe) for s in scores]
    total = sum(s.sum(-1) for s in scores)
    out = torch.zeros_like(q)
    if st["longest"]:
        out = out + torch.matmul(scores[0], values[0])
    if shared:
        p = scores[-1].view(-1, per, hkv, g, case["prefix"]).permute(0, 2, 1, 3, 4).reshape(-1, hkv, per * g, case["prefix"])
        out = out + torch.matmul(p, pv).view(-1, hkv, per, g, dim).permute(0, 2, 1, 3, 4).reshape(n, hkv, g, dim)
    empty = total == 0
    out = out / torch.where(empty, torch.ones_like(total), total).unsqueeze(-1)
    lse = torch.where(empty, torch.full_like(total, -math.inf), safe.squeeze(-1) + torch.log(total))
    return {"out": out.reshape(n, hkv * g, dim).to(torch.bfloat16), "lse": lse.reshape(n, hkv * g)}


def _bits_to_bool(bits, vocab):
    return ((bits.unsqueeze(-1) >> torch.arange(32, device=DEVICE, dtype=torch.int32)) & 1).flatten(-2)[..., :vocab].bool()


def _plain_rules(st):
    vocab, rows = st["case"]["vocab"], st["case"]["rows"]
    x = st["logits"].float()
    live = torch.arange(st["history"].shape[1], device=DEVICE) < st["history_lens"].unsqueeze(1)
    count = torch.zeros((rows, vocab), device=DEVICE).scatter_add_(1, st["history"].long(), live.float())
    seen = (count > 0) | _bits_to_bool(st["prompt_bits"], vocab)[st["prompt_rows"].long()]
    rep = st["repetition"].unsqueeze(1)
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - st["frequency"].unsqueeze(1) * count - st["presence"].unsqueeze(1) * (count > 0).float()
    n = st["bias_indptr"][-1:]
    e = torch.arange(st["bias_ids"].numel(), device=DEVICE)
    row = torch.clamp(torch.searchsorted(st["bias_indptr"], e, right=True) - 1, max=rows - 1)
    value = torch.where(e < n, st["bias_values"], torch.zeros_like(st["bias_values"]))
    bias = torch.zeros(rows * vocab, device=DEVICE).scatter_add_(0, row * vocab + st["bias_ids"].long(), value)
    x = x + bias.view(rows, vocab)
    allowed = _bits_to_bool(st["mask_bits"], vocab)[torch.clamp(st["mask_rows"], min=0).long()] | (st["mask_rows"] < 0).unsqueeze(1)
    return {"logits": torch.where(allowed, x, torch.full_like(x, -math.inf)).to(st["logits"].dtype)}


def _plain_mark(st):
    rows, vocab = st["case"]["rows"], st["case"]["vocab"]
    words = (vocab + 31) // 32
    e = torch.arange(st["ids"].numel(), device=DEVICE)
    row = torch.searchsorted(st["indptr"], e, right=True) - 1
    hit = torch.zeros((rows + 1) * words * 32, dtype=torch.int32, device=DEVICE)
    hit[row * (words * 32) + st["ids"].long()] = 1                         # the entry behind the last row falls into row `rows`
    hit = hit[:rows * words * 32].view(rows, words, 32).long() << torch.arange(32, device=DEVICE)
    word = hit.sum(-1)
    return {"bits": torch.where(word >= 2 ** 31, word - 2 ** 32, word).int()}


# -------------------------------------------------------------------------------------------------------------- work
def work(case):
    op = case["op"]
    if op == "pages":
        n, tokens = case["samples"], case["samples"] * (case["new_lo"] + case["new"]) / 2
        entries = n * _most_entries(case) if case["mode"] == "build" else tokens / PAGE
        # lengths, indptr and indices, a free page for each new page, 8 bytes of slot for each token of the capacity
        return {"bytes": 24.0 * n + 4 * entries + 4 * tokens / PAGE + 8 * n * case["new"], "flops": 0}
    if op == "kv4":
        tokens = case["samples"] * (case["new_lo"] + case["new"]) / 2
        row = case["kv_heads"] * case["dim"]
        # K and V in bf16 read and written once, 5 bits an element written and read
        return {"bytes": tokens * (8.0 * row + 2 * 1.25 * row + 16), "flops": tokens * row * 8}
    if op == "decode":
        n = case["prompts"] * case["samples"]
        own_tokens = n * (case["suffix_lo"] + case["suffix"]) / 2
        shared = int(_prefix_lengths(case).sum())
        row = case["kv_heads"] * case["dim"]
        qrow = case["q_heads"] * case["dim"]
        return {"bytes": own_tokens * 1.25 * row + 4 * own_tokens / PAGE + 4.0 * shared * row + n * (4 * qrow + 4 * case["q_heads"]),
                "flops": 4.0 * qrow * (own_tokens + shared * case["samples"])}
    if op == "rules":
        size = 2 if case["dtype"] == "bf16" else 4
        rows, vocab = case["rows"], case["vocab"]
        return {"bytes": 2.0 * size * rows * vocab + (max(1, rows // 64) + 2) * vocab / 8 + 2 * rows * case["history"] + 4 * rows * case["biases"],
                "flops": 6.0 * rows * vocab}
    return {"bytes": 3.0 * case["rows"] * case["ids"] + case["rows"] * case["vocab"] / 8, "flops": 0}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    op = case["op"]
    if op in ("pages", "mark"):
        return None
    st = prepare(case, seed)
    return {"kv4": _exact_kv4, "decode": _exact_decode, "rules": _exact_rules}[op](st)


def _exact_round_trip(x):
    """What each channel reads back as: 16 levels from the group's lowest value up, their distance a bf16 number."""
    tokens, heads, dim = x.shape
    x = x.double().reshape(tokens, heads, dim // GROUP, GROUP)
    low = x.min(3, keepdim=True).values
    step = ((x.max(3, keepdim=True).values - low) / 15.0).bfloat16().double()
    level = torch.where(step == 0, torch.zeros_like(x), torch.round((x - low) / step))
    return (low + step * torch.clamp(level, 0.0, 15.0)).reshape(tokens, heads, dim)


def _exact_kv4(st):
    got = {}
    for name in ("k", "v"):
        x = _exact_round_trip(st[name])
        x[st["slots"] < 0] = 0.0
        got[name] = x
    return got


def _exact_rows(cells, dim, which):
    """One head's tokens of every page: cells [pages, 20 D] -> [pages, 16, D] float64."""
    codes = cells[:, which * 8 * dim:(which + 1) * 8 * dim]
    params = cells[:, 16 * dim:].contiguous().view(torch.bfloat16).double()
    groups = dim // GROUP
    out = torch.empty((cells.shape[0], PAGE, dim), dtype=torch.float64, device=cells.device)
    for t in range(PAGE):
        mine = params[:, (which * PAGE + t) * 8:][:, :8] if dim == 128 else params[:, t * 8 + which * 4:][:, :4]
        for i in range(groups):
            at = 16 * (t * groups + (i ^ ((t // 2) % 4 if dim == 128 else (t // 4) % 2)))
            pair, scale, low = codes[:, at:at + 16], mine[:, i:i + 1], mine[:, groups + i:groups + i + 1]
            out[:, t, i * GROUP:(i + 1) * GROUP:2] = (pair % 16) * scale + low
            out[:, t, i * GROUP + 1:(i + 1) * GROUP:2] = (pair // 16) * scale + low
    return out


def _exact_decode(st):
    case = st["case"]
    hkv, dim = case["kv_heads"], case["dim"]
    g = case["q_heads"] // hkv
    n = case["prompts"] * case["samples"]
    out = torch.zeros((n, hkv, g, dim), dtype=torch.float64, device=DEVICE)
    lse = torch.full((n, hkv, g), -math.inf, dtype=torch.float64, device=DEVICE)
    first = np.concatenate([[0], np.cumsum(_prefix_lengths(case))])
    indptr, lens = st["page_indptr"].tolist(), st["suffix_lens"].tolist()
    ids = st["page_indices"].long()
    for h in range(hkv):
        keys, vals = (_exact_rows(st["pool"][:, h], dim, i) for i in range(2))
        pk, pv = st["prefix_k"][:, h].double(), st["prefix_v"][:, h].double()
        for s in range(n):
            a, b = first[s // case["samples"]], first[s // case["samples"] + 1]
            mine = ids[indptr[s]:indptr[s + 1]]
            k = torch.cat([pk[a:b], keys[mine].reshape(-1, dim)[:lens[s]]])
            v = torch.cat([pv[a:b], vals[mine].reshape(-1, dim)[:lens[s]]])
            if not k.shape[0]:
                continue
            x = (st["q"][s, h * g:(h + 1) * g].double() @ k.T) / math.sqrt(dim)
            lse[s, h] = torch.logsumexp(x, 1)
            out[s, h] = torch.softmax(x, 1) @ v
    return {"out": out.view(n, -1, dim), "lse": lse.view(n, -1)}


def _exact_rules(st):
    rows, vocab = st["case"]["rows"], st["case"]["vocab"]
    host = {k: v.cpu() for k, v in st.items() if isinstance(v, torch.Tensor)}
    words = {k: host[k].numpy().view(np.uint32) for k in ("prompt_bits", "mask_bits")}
    result = np.empty((rows, vocab))
    column = np.arange(vocab)
    for r in range(rows):
        x = host["logits"][r].double().numpy().copy()
        said = host["history"][r, :int(host["history_lens"][r])].numpy()
        count = np.bincount(said, minlength=vocab)[:vocab].astype(np.float64)
        in_prompt = (words["prompt_bits"][int(host["prompt_rows"][r])][column // 32] >> (column % 32).astype(np.uint32)) & 1
        rep = float(host["repetition"][r])
        hit = (count > 0) | (in_prompt > 0)
        x[hit] = np.where(x[hit] > 0, x[hit] / rep, x[hit] * rep)
        x -= float(host["frequency"][r]) * count
        x[count > 0] -= float(host["presence"][r])
        a, b = int(host["bias_indptr"][r]), int(host["bias_indptr"][r + 1])
        np.add.at(x, host["bias_ids"][a:b].numpy(), host["bias_values"][a:b].double().numpy())
        if int(host["mask_rows"][r]) >= 0:
            allowed = (words["mask_bits"][int(host["mask_rows"][r])][column // 32] >> (column % 32).astype(np.uint32)) & 1
            x[allowed == 0] = -np.inf
        result[r] = x
    return {"logits": torch.from_numpy(result)}
