"""Definitions of the operators over a bf16 cache in pages, written out in 64 bits: attention of new tokens, the weight cached tokens
receive, eviction of pages by that weight.  One sample, one head and one row at a time; nothing is shared with the kernels."""
import numpy as np

PAGE = 16


def tokens_of(pool, page_list, head, length):
    """The first `length` rows of a sample's list for one KV head: [length, D] float64 (pool: [pages, heads, 16, D] float)."""
    if not length:
        return np.zeros((0, pool.shape[-1]))
    pages = np.asarray(page_list)[:-(-length // PAGE)]
    return np.concatenate([pool[p, head] for p in pages]).astype(np.float64)[:length]


def attend(q, k_pool, v_pool, page_indptr, page_indices, kv_lens, q_indptr, sm_scale, prior_out=None, prior_lse=None):
    """(out [T, Hq, D], lse [T, Hq], size [T, Hq, D]): size is sum_j weight_j |v_j|, the scale of rounding errors in the weights.  Rows of no
    sample come out as NaN."""
    T, Hq, D = q.shape
    group = Hq // k_pool.shape[1]
    out, lse, size = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan), np.full((T, Hq, D), np.nan)
    for s, length in enumerate(kv_lens):
        a, b = int(q_indptr[s]), int(q_indptr[s + 1])
        pages = page_indices[page_indptr[s]:page_indptr[s + 1]]
        for head in range(k_pool.shape[1]):
            k, v = (tokens_of(p, pages, head, int(length)) for p in (k_pool, v_pool))
            for row in range(a, b):
                seen = max(0, int(length) - (b - a) + (row - a) + 1)
                for h in range(head * group, (head + 1) * group):
                    if not seen:
                        out[row, h], lse[row, h], size[row, h] = 0.0, -np.inf, 0.0
                        continue
                    x = (k[:seen] @ q[row, h].astype(np.float64)) * sm_scale
                    top = x.max()
                    w = np.exp(x - top)
                    total = w.sum()
                    out[row, h] = (w[:, None] * v[:seen]).sum(0) / total
                    size[row, h] = (w[:, None] * np.abs(v[:seen])).sum(0) / total
                    lse[row, h] = top + np.log(total)
    if prior_out is not None:
        for row in range(T):
            for h in range(Hq):
                p = float(prior_lse[row, h])
                if np.isnan(lse[row, h]) or (p == -np.inf and lse[row, h] == -np.inf):
                    continue
                both = np.logaddexp(p, lse[row, h])
                mine, other = np.exp(lse[row, h] - both), np.exp(p - both)
                out[row, h] = mine * out[row, h] + (other * prior_out[row, h].astype(np.float64) if other else 0.0)
                size[row, h] = mine * size[row, h]
                lse[row, h] = both
    return out, lse, size


def accumulate(weights, q, lse, k_pool, page_indptr, page_indices, kv_lens, q_indptr, sm_scale):
    """The array [pages, heads, 16] after a call, float64: cells of samples with new tokens get their sums, the new tokens' own from zero."""
    got = weights.astype(np.float64)
    group = q.shape[1] // k_pool.shape[1]
    for s, length in enumerate(kv_lens):
        a, b = int(q_indptr[s]), int(q_indptr[s + 1])
        pages = page_indices[page_indptr[s]:page_indptr[s + 1]]
        if a == b:
            continue
        for head in range(k_pool.shape[1]):
            k = tokens_of(k_pool, pages, head, int(length))
            for j in range(int(length)):
                total = 0.0 if j >= int(length) - (b - a) else float(weights[pages[j // PAGE], head, j % PAGE])
                first = max(a, a + j - (int(length) - (b - a)))
                x = (q[first:b, head * group:(head + 1) * group].astype(np.float64) @ k[j]) * sm_scale - lse[first:b, head * group:(head + 1) * group]
                got[pages[j // PAGE], head, j % PAGE] = total + np.exp(x).sum()
    return got


def evict(weights, page_indptr, page_indices, kv_lens, budgets, recent, free_pages, free_count):
    """(page_indices, kv_lens, free_pages, free_count) after a call."""
    out, lens, stack = np.array(page_indices), np.array(kv_lens), [int(p) for p in free_pages[:free_count]]
    for s, length in enumerate(kv_lens):
        held = -(-int(length) // PAGE)
        mine = [int(p) for p in page_indices[page_indptr[s]:page_indptr[s] + held]]
        budget = int(budgets[s])
        if held <= budget:
            continue
        newest = min(recent, budget)
        older = list(range(held - newest))
        heavy = [np.nanmax(np.where(np.isnan(weights[p]), -np.inf, weights[p])) + 0.0 for p in mine]
        stay = sorted(sorted(older, key=lambda i: (-heavy[i], i))[:budget - newest]) + list(range(held - newest, held))
        keep = set(stay)
        stack += [mine[i] for i in older if i not in keep]
        out[page_indptr[s]:page_indptr[s] + held] = [mine[i] for i in stay] + [-1] * (held - budget)
        lens[s] = int(length) - PAGE * (held - budget)
    free = np.array(free_pages)
    free[:len(stack)] = stack
    return out, lens, free, len(stack)
