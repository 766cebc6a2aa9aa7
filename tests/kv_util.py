"""Caches on the device beside the oracle's, for the tests of the key/value cache."""
import numpy as np
import torch

import paper_2511_04063_b200 as dq
from oracle import kv_cache as kv

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def put(x, dtype):
    return torch.from_numpy(np.asarray(x)).cuda().to(dtype)


def table_of(rng, lengths, page, spare=2, width=None):
    """Pages in no order: (table, number of pages)."""
    need = [max(0, -(-n // page)) for n in lengths]
    width = width or max(need + [1])
    order = rng.permutation(sum(need) + spare)
    table, at = np.full((len(lengths), width), -1), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


def filled(rng, lengths, heads, dim, page, spread=1.0, fill=255, width=None):
    """(oracle cache, device cache) with keys and values in all slots below the lengths; everything else is `fill` (255: a NaN)."""
    table, n_pages = table_of(rng, lengths, page, width=width)
    c = kv.Cache(n_pages, heads, dim, page, table, lengths, fill)
    for b, n in enumerate(lengths):
        for h in range(heads):
            mean = rng.standard_normal(dim)
            for slot in range(max(0, min(n, table.shape[1] * page))):
                c.write(b, h, slot, 0, spread * rng.standard_normal(dim) + mean)
                c.write(b, h, slot, 1, spread * rng.standard_normal(dim) * np.exp(0.5 * rng.standard_normal()))
    return c, on_device(c)


def on_device(c):
    return dq.dq_kv_cache(torch.from_numpy(c.pages).cuda(), torch.from_numpy(c.table.astype(np.int32)).cuda(),
                          torch.from_numpy(c.lengths.astype(np.int32)).cuda(), c.dim)


def starts_of(queries):
    return torch.tensor(np.concatenate(([0], np.cumsum(queries))), dtype=torch.int32, device="cuda")


def workspace(dim):
    return torch.zeros(dq.dq_kv_attention_workspace(dim), dtype=torch.uint8, device="cuda")


def attend(cache, q, scale, starts=None, work=None, out=None, lse=None):
    """(out, lse) of dq_kv_attention, filled with a number that the call has to overwrite."""
    out = torch.full(q.shape, 77.0, dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full(q.shape[:2], 77.0, device="cuda") if lse is None else lse
    dq.dq_kv_attention(q, cache, scale, out, workspace(cache.head_dim) if work is None else work, starts=starts, lse=lse)
    assert dq.dq_mx_status() == dq.DQ_OK
    return out, lse


def logit_bound(logits, dim):
    """A logit is a sum of dim exact products (a code's four bits times a query's 8 or 11; queries below 2^-24 of their row's largest are
    off by 2^-35 of it) in fp32, in steps that may truncate, times a scale, plus an offset times the sum of the query: off by at most (dim / 16 + 24) 2^-23 of the magnitudes' sum."""
    return (dim / 16 + 24) * 2.0 ** -23 * logits + 2.0 ** -22


def check_attention(c, b, q, first, n, group, scale, out, lse):
    """Rows first .. first + n of out and lse against the oracle.  p = exp(S - top) / l is off by twice the logits' error relatively
    (S and l), by 2^-20 for the exponentials, sums and joins, and by half an fp16 step, 2^-11, where it is rounded for the product:
    of a term that is at least 2^-20 of what a key with p = 1 and the largest scale of its stage has (2^6 .. 2^7, fp16's normal numbers
    begin at 2^-14), else by 2^-25 / 2^6 of the latter.  For many rows the values are rounded to fp16 too: by 2^-11, or 2^-25 where the
    largest scale is above 2^-10 (2^-15 of it, 2^-17 of the largest value: a scale is at most 2/15 of that).  The output is then rounded
    once."""
    dtype = q.dtype
    for h in range(c.heads):
        heads = slice(h * group, (h + 1) * group)
        r = kv.attention(c, b, h, f64(q[first:first + n, heads]), scale)
        e = logit_bound(r["logits"], c.dim)
        got = f64(lse[first:first + n, heads])
        empty = np.isneginf(r["lse"])
        assert (np.isneginf(got) == empty).all()
        full = ~empty
        assert (np.abs(got[full] - r["lse"][full]) <= e[full] + 2.0 ** -21 * (1 + np.abs(r["lse"][full]))).all()
        bound = (2 * e[..., None] + 2.0 ** -20 + 2 * 2.0 ** -11) * r["terms"] * 1.01 + UNIT[dtype] * np.abs(r["out"]) * 1.01 + LEAST[dtype]
        bound += (c.length(b) * 2.0 ** -31 + 2.0 ** -17) * r["largest"]
        got = f64(out[first:first + n, heads])
        assert (np.abs(got - r["out"]) <= bound).all(), float((np.abs(got - r["out"]) / bound).max())
