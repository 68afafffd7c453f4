"""The 4-bit K/V cache in plain numpy: quantisation of a group, the cell layout byte by byte, and attention in fp64 over the
values the cells stand for."""
from __future__ import annotations

import math

import numpy as np

PAGE, GROUP = 16, 32


def bf16_to_f64(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def f64_to_bf16(x):
    """Round to nearest even; x must be exact in fp32 or far from a bf16 rounding border."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = ((u + (np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1)))) >> np.uint32(16)).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def f64_to_bf16_once(x):
    """fp64 -> bf16 bits in one rounding to nearest even (to odd in fp32 first, which keeps every tie and every side of it)."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        f = x.astype(np.float32)
        toward = np.where(np.abs(f.astype(np.float64)) > np.abs(x), np.nextafter(f, np.float32(0)), f)       # truncated
        inexact = np.isfinite(x) & (toward.astype(np.float64) != x)
        u = toward.view(np.uint32) | inexact.astype(np.uint32)
    return f64_to_bf16(u.view(np.float32))


def quantise(bits):
    """bits [..., D] bf16 -> (codes [..., D] uint8, scale and offset bf16 bits [..., D / 32])."""
    with np.errstate(all="ignore"):
        x = bf16_to_f64(bits)
        g = x.reshape(*x.shape[:-1], -1, GROUP)
        low, high = g.min(-1), g.max(-1)
        scale_bits = f64_to_bf16((high - low).astype(np.float32) / np.float32(15))
        scale = bf16_to_f64(scale_bits)
        bad = ~np.isfinite(scale)
        scale_bits = np.where(bad, np.uint16(0x7FC0), scale_bits)
        t = np.rint((g - low[..., None]).astype(np.float32) / scale[..., None].astype(np.float32))
        codes = np.where((scale[..., None] > 0) & ~bad[..., None], np.clip(t, 0, 15), 0)
    return np.nan_to_num(codes).astype(np.uint8).reshape(x.shape), scale_bits, f64_to_bf16(low)


def values(codes, scale_bits, offset_bits):
    with np.errstate(invalid="ignore"):
        g = codes.reshape(*codes.shape[:-1], -1, GROUP).astype(np.float64)
        return (g * bf16_to_f64(scale_bits)[..., None] + bf16_to_f64(offset_bits)[..., None]).reshape(codes.shape)


def cell_bytes(D):
    return 20 * D


def chunk_at(D, t, g):
    return 16 * (t * (D // GROUP) + (g ^ ((t // 2) % 4 if D == 128 else (t // 4) % 2)))


def params_at(D, which, t):
    return 16 * D + (which * 256 + t * 16 if D == 128 else t * 16 + which * 8)


def write_token(cell, t, k_bits, v_bits):
    """cell [20 D] uint8 (modified): token t of the page."""
    D = cell.size // 20
    for which, bits in ((0, k_bits), (1, v_bits)):
        codes, s, b = quantise(bits)
        for g in range(D // GROUP):
            at = which * 8 * D + chunk_at(D, t, g)
            c = codes[g * GROUP:(g + 1) * GROUP]
            cell[at:at + 16] = c[0::2] | (c[1::2] << 4)
        at = params_at(D, which, t)
        cell[at:at + 4 * (D // GROUP)] = np.concatenate([s, b]).astype(np.uint16).view(np.uint8)


def read_token(cell, t):
    """(K parts, V parts), each (codes [D], scale bits [D/32], offset bits [D/32])."""
    D = cell.size // 20
    out = []
    for which in (0, 1):
        codes = np.empty(D, np.uint8)
        for g in range(D // GROUP):
            at = which * 8 * D + chunk_at(D, t, g)
            codes[g * GROUP:(g + 1) * GROUP:2] = cell[at:at + 16] & 15
            codes[g * GROUP + 1:(g + 1) * GROUP:2] = cell[at:at + 16] >> 4
        at = params_at(D, which, t)
        p = cell[at:at + 4 * (D // GROUP)].copy().view(np.uint16)
        out.append((codes, p[:D // GROUP], p[D // GROUP:]))
    return out


def store(pool, slots, k_bits, v_bits):
    """pool [pages, Hkv, 20 D] uint8 (modified); skips negative slots and slots beyond the pool."""
    for i, slot in enumerate(slots):
        if 0 <= slot < pool.shape[0] * PAGE:
            for h in range(pool.shape[1]):
                write_token(pool[slot // PAGE, h], int(slot) % PAGE, k_bits[i, h], v_bits[i, h])


def random_pool(pages, heads, D, seed):
    """Cells of N(0, 1) rows, made in bulk (the layout of write_token)."""
    rng = np.random.default_rng(seed)
    pool = np.zeros((pages, heads, cell_bytes(D)), np.uint8)
    for which in (0, 1):
        codes, s, b = quantise(f64_to_bf16(rng.standard_normal((pages, heads, PAGE, D)).astype(np.float32)))
        packed = codes[..., 0::2] | (codes[..., 1::2] << 4)
        for t in range(PAGE):
            for g in range(D // GROUP):
                at = which * 8 * D + chunk_at(D, t, g)
                pool[:, :, at:at + 16] = packed[:, :, t, g * 16:(g + 1) * 16]
            at = params_at(D, which, t)
            pool[:, :, at:at + 4 * (D // GROUP)] = np.concatenate([s, b], -1)[:, :, t].astype(np.uint16).view(np.uint8)
    return pool


def pool_values(pool, which):
    """pool [pages, Hkv, 20 D] -> (codes - 8, scale, offset + 8 scale) as fp64 [pages, Hkv, 16, D]."""
    D = pool.shape[-1] // 20
    NG = D // GROUP
    codes = np.empty((*pool.shape[:2], PAGE, D))
    s = np.empty((*pool.shape[:2], PAGE, NG))
    b = np.empty_like(s)
    for t in range(PAGE):
        for g in range(NG):
            at = which * 8 * D + chunk_at(D, t, g)
            c = pool[:, :, at:at + 16]
            codes[:, :, t, g * GROUP:(g + 1) * GROUP:2] = c & 15
            codes[:, :, t, g * GROUP + 1:(g + 1) * GROUP:2] = c >> 4
        at = params_at(D, which, t)
        p = np.ascontiguousarray(pool[:, :, at:at + 4 * NG]).view(np.uint16)
        s[:, :, t], b[:, :, t] = bf16_to_f64(p[..., :NG]), bf16_to_f64(p[..., NG:])
    s, b = np.repeat(s, GROUP, -1), np.repeat(b, GROUP, -1)
    return codes - 8, s, b + 8 * s


def attend(w):
    """Decode attention in fp64.  w: psa_workloads fields, with `kv4_pool` [pages, Hkv, 20 D] uint8 in place of the bf16 pools.
    Returns (out [B, Hq, D], lse [B, Hq], out_scale [B, Hq, D], lse_scale [B, Hq]): the last two are the magnitudes rounding
    errors are relative to -- sum_t weight_t (|s (code - 8)| + |b + 8 s|) over the sample's own tokens plus sum_t weight_t |v_t| over
    the shared ones, and the largest sum of absolute terms of a score."""
    B, Hq, D = w["q"].shape
    Hkv = w["num_kv_heads"]
    G = Hq // Hkv
    q = bf16_to_f64(w["q"])
    pk, pv = bf16_to_f64(w["prefix_k"]), bf16_to_f64(w["prefix_v"])
    K, V = pool_values(w["kv4_pool"], 0), pool_values(w["kv4_pool"], 1)
    tok = np.concatenate([[0], np.cumsum(w["prefix_lens"])])
    of = np.repeat(np.arange(len(w["n_samples"])), w["n_samples"])
    out, lse = np.zeros((B, Hq, D)), np.full((B, Hq), -np.inf)
    out_scale, lse_scale = np.zeros((B, Hq, D)), np.zeros((B, Hq))
    for b in range(B):
        S = int(w["suffix_lens"][b])
        ids = w["page_indices"][w["page_indptr"][b]:w["page_indptr"][b] + (S + PAGE - 1) // PAGE]
        for h in range(Hkv):
            take = lambda x: x[ids, h].reshape(-1, D)[:S]  # noqa: E731
            kc, ks, kb = (take(x) for x in K)
            vc, vs, vb = (take(x) for x in V)
            a, e = tok[of[b]], tok[of[b] + 1]
            keys = np.concatenate([pk[a:e, h], ks * kc + kb])
            vals = np.concatenate([pv[a:e, h], vs * vc + vb])
            if not len(keys):
                continue
            mag_v = np.concatenate([np.abs(pv[a:e, h]), np.abs(vs * vc) + np.abs(vb)])
            for r in range(G):
                x = q[b, h * G + r]
                score = keys @ x * w["sm_scale"]
                m = score.max()
                p = np.exp(score - m)
                z = p.sum()
                out[b, h * G + r] = p @ vals / z
                lse[b, h * G + r] = m + math.log(z)
                out_scale[b, h * G + r] = p @ mag_v / z
                group_sum = np.repeat(x.reshape(-1, GROUP).sum(1), GROUP) / GROUP
                mag = np.concatenate([np.abs(pk[a:e, h]) @ np.abs(x), (np.abs(ks) * (kc + 8)) @ np.abs(x) + np.abs(kb - 8 * ks) @ np.abs(group_sum)])
                lse_scale[b, h * G + r] = mag.max() * w["sm_scale"]
    return out, lse, out_scale, lse_scale
