"""Paged stores and their attention in 64 bits, for the tests: plain numpy, element by element where it matters."""
import numpy as np
import torch

D = 128


def pack(codes, bits):
    """Integer codes [..., 128] -> int32 words [..., 128 * bits / 32]."""
    per = 32 // bits
    c = np.asarray(codes, dtype=np.uint64).reshape(*codes.shape[:-1], D // per, per)
    words = np.zeros(c.shape[:-1], dtype=np.uint64)
    for i in range(per):
        words |= c[..., i] << np.uint64(bits * i)
    return words.astype(np.uint32).view(np.int32)


def unpack(words, bits):
    w = np.ascontiguousarray(words).view(np.uint32)
    out = np.empty((*w.shape[:-1], D), dtype=np.int64)
    for c in range(D):
        out[..., c] = (w[..., c * bits // 32] >> np.uint32(c * bits % 32)) & np.uint32((1 << bits) - 1)
    return out


def values(words, meta, bits):
    """float64 [..., 128] that words and (scale, zero) float16 [..., groups, 2] stand for."""
    g = D // meta.shape[-2]
    with np.errstate(invalid="ignore"):
        return unpack(words, bits) * np.repeat(meta[..., 0].astype(np.float64), g, -1) + np.repeat(meta[..., 1].astype(np.float64), g, -1)


def quantize(x, bits, group):
    """codes int64, meta float16 of float64 [..., 128] by the definition of squat_paged_write."""
    g = x.reshape(*x.shape[:-1], D // group, group)
    top = (1 << bits) - 1
    low, high = g.min(-1), g.max(-1)
    zero = low.astype(np.float32).astype(np.float16)
    scale = ((high - low) / top).astype(np.float32).astype(np.float16)
    s = scale.astype(np.float64)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        codes = np.clip(np.rint((g - zero.astype(np.float64)[..., None]) / s), 0, top)
    codes = np.where(s > 0, codes, 0).astype(np.int64)
    return codes.reshape(x.shape), np.stack([scale, zero], -1)


def random_store(rng, n_pages, heads, page, bits, group, scale=1.0):
    """Codes and meta (numpy) of a store in which every page holds something."""
    codes = rng.integers(0, 1 << bits, (n_pages, heads, page, D))
    step = (rng.uniform(0.5, 1.5, (n_pages, heads, page, D // group)) * 4 * scale / (1 << bits)).astype(np.float16)
    zero = (-2 * scale * rng.uniform(0.7, 1.3, step.shape)).astype(np.float16)
    return pack(codes, bits), np.stack([step, zero], -1)


def lists(rng, lens, page, n_pages, width=None):
    """A page list per sequence, drawn without repetition; unused entries hold a number that is no page."""
    need = [-(-n // page) for n in lens]
    order = rng.permutation(n_pages)[:sum(need)]
    table = np.full((len(lens), width or max(max(need), 1)), 0x7FFFFFFF, dtype=np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table


def attention(q, store, bits, table, lens, starts, out_scale, rounded_keys=False):
    """(out, lse, sum p |v|, and the bound's logit error) in float64.  q [n, Hq, 128] float64; store (kc, km, vc, vm) numpy.  A page number
    outside the store: its tokens are seen by nobody.  rounded_keys: the keys enter rounded to fp16, 2^-11 of each product."""
    kc, km, vc, vm = store
    n_pages, heads, page = kc.shape[:3]
    qpk = q.shape[1] // heads
    bias = {2: 16, 4: 64, 8: 1024}[bits]
    out, lse, mass, off = np.zeros(q.shape), np.full(q.shape[:2], -np.inf), np.zeros(q.shape), np.zeros(q.shape[:2])
    for s, length in enumerate(lens):
        a, b = int(starts[s]), int(starts[s + 1])
        ids = table[s][:-(-length // page)] if length > 0 else table[s][:0]
        there = np.repeat((ids >= 0) & (ids < n_pages), page)[:length]
        ids = np.where((ids >= 0) & (ids < n_pages), ids, 0)
        for h in range(heads):
            k = values(kc[ids, h].reshape(-1, kc.shape[-1]), km[ids, h].reshape(-1, *km.shape[-2:]), bits)[:length]
            v = values(vc[ids, h].reshape(-1, vc.shape[-1]), vm[ids, h].reshape(-1, *vm.shape[-2:]), bits)[:length]
            size = np.repeat(np.abs(km[ids, h].reshape(-1, *km.shape[-2:])[:length].astype(np.float64)) * [(bias + (1 << bits)), 1.0], D // km.shape[-2], -2).sum(-1)
            for j in range(h * qpk, (h + 1) * qpk):
                if length <= 0 or b == a:
                    continue
                qj = q[a:b, j]
                seen = there & (np.arange(length) <= length - (b - a) + np.arange(b - a)[:, None])
                x = np.where(seen, out_scale * (qj @ k.T), -np.inf)
                some = seen.any(1)
                m = np.where(some, x.max(1), 0.0)
                p = np.exp(x - m[:, None])
                total = p.sum(1)
                p = p / np.where(some, total, 1.0)[:, None]
                with np.errstate(divide="ignore"):
                    lse[a:b, j] = np.where(some, m + np.log(total), -np.inf)
                out[a:b, j], mass[a:b, j] = p @ v, p @ np.abs(v)
                # a logit: 128 products summed in fp32 from the bias on, then a handful of operations a group
                worst = lambda y: np.where(seen, y, 0.0).max(1)       # noqa: E731
                off[a:b, j] = abs(out_scale) * worst(np.abs(qj) @ size.T) * 40 * 2.0 ** -24 + worst(np.abs(x)) * 2.0 ** -22
                if rounded_keys:
                    off[a:b, j] += abs(out_scale) * worst(np.abs(qj) @ np.abs(k).T) * 2.0 ** -11
    return out, lse, mass, off


def to_device(store):
    return [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in store]
