"""The operators around the 4-bit key/value cache where their parts meet: rows, keys and scales of zero behind a mask, scales far apart,
long axes that one CTA goes over, batches of decoding sequences and a chunk, missing pages in eviction.  Against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2511_04063_b200 as dq
from kv_util import UNIT, attend, check_attention, f64, filled, logit_bound, on_device, put, starts_of, table_of
from oracle import kv_cache as kv
from test_gpu_kv import attention_case, weights_case

pytestmark = pytest.mark.gpu

DIMS = (64, 128, 256)
# One sequence of so few query rows that its keys are cut between CTAs where the table is wide, and where it is not one CTA goes
# over all of them.
WIDE, NARROW = 2048, None


def chunk_rows(dim):
    """Queries of two heads, enough for the kernel of many rows."""
    return 140 if dim == 256 else 90


def check_all(c, cache, q, scale, queries):
    out, lse = attend(cache, q, scale, starts_of(queries))
    group, first = q.shape[1] // c.heads, 0
    for b, n in enumerate(queries):
        check_attention(c, b, q, first, n, group, scale, out, lse)
        first += n


@pytest.mark.parametrize("slots", (NARROW, WIDE))
@pytest.mark.parametrize("dim", DIMS)
def test_a_prompt_of_zeros(dim, slots):
    """Queries, keys and values are zero, as in a pass over padding: every output is zero, a token's lse the logarithm of what it sees."""
    n = 150
    table, n_pages = table_of(np.random.default_rng(dim), [n], 16, width=slots and slots // 16)
    c = kv.Cache(n_pages, 2, dim, 16, table, [n], 0xff)
    cache = on_device(c)
    zeros = torch.zeros((n, 4, dim), dtype=torch.bfloat16, device="cuda")
    dq.dq_kv_append(zeros[:, :2], zeros[:, 2:], cache)
    for queries in (n, 1):                                       # by both kernels
        out, lse = attend(cache, zeros[:queries], 0.1)
        sees = torch.arange(n - queries + 1, n + 1, dtype=torch.float64, device="cuda")
        assert bool((out == 0).all())
        assert float((lse.double() - sees.log()[:, None]).abs().max()) <= 2.0 ** -20 * (1 + np.log(n))   # (an exponential's and a logarithm's error)
        weights = torch.full((1, 2, cache.slots), 77.0, device="cuda")
        dq.dq_kv_attention_weights(zeros[:queries], lse, cache, 0.1, weights)
        assert bool(torch.isfinite(weights[..., :n]).all()) and bool((weights[..., n:] == 77).all())
        assert float((weights[..., :n].double().sum(-1) - 2 * queries).abs().max()) <= 2 * queries * 2.0 ** -16   # (lse's error, and as much again)


@pytest.mark.parametrize("slots", (NARROW, WIDE))
@pytest.mark.parametrize("dim", DIMS)
def test_zero_queries_over_keys_without_a_range_behind_a_mask(dim, slots):
    """Keys that are one number each in the tile that the causal mask cuts, in the last tile, which the length cuts, and beside pages that
    are missing; some query rows of zeros among others that are not, and values of a row's own size."""
    rng = np.random.default_rng(dim + 1)
    n, length = chunk_rows(dim), 300
    for level in (0.0, 0.4, -3.0, 100.0):
        c, _ = filled(rng, [length], 1, dim, 16, width=slots and slots // 16)
        c.table[0, [1, 17]] = -1                                 # a tile has a hole before the queries, another among them
        for slot in range(length):
            c.write(0, 0, slot, 0, np.full(dim, level))
        q = rng.standard_normal((n, 2, dim))
        q[::3], q[1::3, 1] = 0.0, 0.0
        check_all(c, on_device(c), put(q, torch.bfloat16), 0.1, [n])


@pytest.mark.parametrize("slots", (NARROW, WIDE))
@pytest.mark.parametrize("dim", DIMS)
def test_zero_queries_over_a_tile_without_pages(dim, slots):
    rng = np.random.default_rng(dim + 2)
    n, length = chunk_rows(dim), 400
    c, _ = filled(rng, [length], 1, dim, 16, width=slots and slots // 16)
    c.table[0, 8:16] = -1
    q = rng.standard_normal((n, 2, dim))
    q[::2] = 0.0
    check_all(c, on_device(c), put(q, torch.float16), 0.1, [n])
    c.table[0] = -1                                              # none at all
    out, lse = attend(on_device(c), put(q, torch.float16), 0.1)
    assert bool((out == 0).all()) and bool((lse == -torch.inf).all())


@pytest.mark.parametrize("slots", (NARROW, WIDE))
@pytest.mark.parametrize("dim", DIMS)
def test_a_scale_of_zero(dim, slots):
    """All that is seen counts alike, whatever the keys: zeros, ordinary ones, large ones."""
    rng = np.random.default_rng(dim + 3)
    n, length = chunk_rows(dim), 200
    for size in (0.0, 1.0, 1e33):
        c, _ = filled(rng, [length], 1, dim, 16, width=slots and slots // 16)
        for slot in range(length):
            c.write(0, 0, slot, 0, size * rng.standard_normal(dim))
        q = put(rng.standard_normal((n, 2, dim)), torch.bfloat16)
        check_all(c, on_device(c), q, 0.0, [n])
        check_all(c, on_device(c), q[-1:], 0.0, [1])


@pytest.mark.parametrize("slots", (NARROW, WIDE))
@pytest.mark.parametrize("dim", DIMS)
def test_large_keys_and_values(dim, slots):
    """Keys of 1e36 with queries of 1e-36, so that the logits are ordinary ones, and values whose means are in bf16's range."""
    rng = np.random.default_rng(dim + 4)
    n, length = chunk_rows(dim), 300
    c, _ = filled(rng, [length], 1, dim, 16, width=slots and slots // 16)
    for slot in range(length):
        c.write(0, 0, slot, 0, 1e36 * rng.standard_normal(dim))
        c.write(0, 0, slot, 1, (1e35 if slot % 3 else 2e36) * rng.standard_normal(dim))
    q = put(1e-36 * rng.standard_normal((n, 2, dim)), torch.bfloat16)
    check_all(c, on_device(c), q, 0.1, [n])
    c.lengths[:] = 40                                            # (few rows: values times exponentials are added before the division)
    check_all(c, on_device(c), q[-2:], 0.1, [2])


@pytest.mark.parametrize("slots", (NARROW, WIDE))
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("apart", (1, 4, 8))
def test_scales_far_apart_in_a_tile(apart, dim, slots):
    """Keys and values next to some with scales 2^(apart + 4) times theirs or so, which a query does not see yet, or sees with a probability of zero.  An
    element of a tile of keys is off by up to 2^-14 of the tile's largest scale, which is held at 2^-10 or more (half of fp16's least step, 2^-25,
    twice: offset and sum), but by nothing where its scale is within 2^-7 of that (8 bits and 3, 2^-10-7-7 = 2^-24); that enters a
    logit with the sum of the query's magnitudes.  An element of a value is off by 2^-14 of the largest scale up to there beside its
    own roundings."""
    rng = np.random.default_rng(dim + apart)
    n, length, big, group, scale = chunk_rows(dim), 250, 2.0 ** apart, 2, 0.1
    c, _ = filled(rng, [length], 1, dim, 16, width=slots and slots // 16)
    q = rng.standard_normal((n, group, dim))
    q[..., 0] = 4.0
    large = [130, length - 2, length - 1]                        # the first one's logit is far below the others'
    for slot in range(length):
        k, v = rng.standard_normal(dim), rng.standard_normal(dim)
        c.write(0, 0, slot, 0, k if slot not in large else big * np.r_[-4.0 * (20 + dim ** 0.5), k[1:] * 0.25])
        c.write(0, 0, slot, 1, v if slot not in large else 32.0 * big * v)
    q = put(q, torch.bfloat16)
    largest = [max(c.raw(0, 0, slot, which)[1] for slot in large) for which in (0, 1)]
    smallest = min(c.raw(0, 0, slot, 0)[1] for slot in range(length))
    held = 0.0 if smallest >= 2.0 ** -6 * largest[0] else 2.0 ** -14 * largest[0]      # (of two scales' powers of two)
    k_terms, v_terms = (c.exact(0, 0, length, which)[1] for which in (0, 1))
    for rows in (q, q[-3:]):                                     # by both kernels
        out, lse = attend(on_device(c), rows, scale)
        r = kv.attention(c, 0, 0, f64(rows), scale)
        for i in range(len(rows) - 2):                           # (the last two see one or both of the others)
            seen = np.arange(length) < length - len(rows) + i + 1
            seen[large[0]] = False
            for g in range(group):
                assert r["p"][i, g, large].max() < 1e-30
                x = np.abs(f64(rows[i, g]))
                e = logit_bound((k_terms[seen] @ x).max() * scale, dim) + held * x.sum() * scale
                assert abs(float(lse[i, g]) - r["lse"][i, g]) <= e + 2.0 ** -21 * (1 + abs(r["lse"][i, g]))
                bound = (np.expm1(2 * e) + 2.0 ** -20 + 2 * 2.0 ** -11) * (r["p"][i, g] @ v_terms) * 1.01
                bound += UNIT[q.dtype] * np.abs(r["out"][i, g]) * 1.01 + 2.0 ** -14 * largest[1]
                assert (np.abs(f64(out[i, g]) - r["out"][i, g]) <= bound).all()


@pytest.mark.parametrize("dim", DIMS)
def test_many_items_over_a_long_axis(dim):
    """More items than SMs, so none is cut: each CTA goes over 21 to 24 tiles of keys, with maxima and the values' largest scale that go on growing.
    One query head of each kv head's is checked, at all of its tokens."""
    rng = np.random.default_rng(dim + 5)
    n, length, heads, group = 300, 3000, 2, 32 if dim == 256 else 64
    c, _ = filled(rng, [1], heads, dim, 64, width=47)
    c.lengths[:] = length
    c.table[0] = rng.permutation(47)
    c.pages = np.full((47, heads, 64 * (dim + 8)), 255, np.uint8)
    for slot in range(length):
        for h in range(heads):
            c.write(0, h, slot, 0, (1 + 3 * slot / length) * rng.standard_normal(dim))
            c.write(0, h, slot, 1, 2.0 ** (slot // 500) * rng.standard_normal(dim))
    cache = on_device(c)
    q = put(2 * rng.standard_normal((n, heads * group, dim)), torch.bfloat16)
    out, lse = attend(cache, q, dim ** -0.5)
    for one in (0, group - 1):
        heads_of = [one, group + one]
        check_attention(c, 0, q[:, heads_of], 0, n, 1, dim ** -0.5, out[:, heads_of], lse[:, heads_of])


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("decoding,chunk", [(40, 30), (5, 400)])
def test_decoding_sequences_and_a_chunk(decoding, chunk, dim):
    """Sequences of one query and one of many in a call: by the kernels for few rows and for many."""
    lengths = [(37 * i) % 150 + 1 for i in range(decoding)]
    at = decoding // 2
    queries = [1] * at + [chunk] + [1] * (decoding - at)
    lengths = lengths[:at] + [chunk + 70] + lengths[at:]
    attention_case(dim, lengths, queries, 1, 4, dim, 32, torch.bfloat16)
    weights_case(dim, lengths, queries, 1, 4, dim, 32, torch.float16)


# ------------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("missing", [(4,), (0,), (2, 3, 5), (1, 4, 6), (0, 1, 2, 3, 4, 5, 6)])
@pytest.mark.parametrize("in_place", (False, True))
def test_evict_where_the_table_names_no_page(missing, in_place):
    """Pages are missing where slots move from, where they move to, at both ends: what has a page is the token that its position says."""
    rng = np.random.default_rng(sum(missing))
    length, keep, recent, heads, dim, page = 108, 40, 8, 2, 64, 16
    c, _ = filled(rng, [length, length], heads, dim, page)
    c.table[0, list(missing)] = [-1, len(c.pages), -9, -1, -1, -1, -1][:len(missing)]   # (the other sequence has all of its pages)
    cache = on_device(c)
    shape = (2, heads, cache.slots)
    weights = rng.exponential(size=shape).astype(np.float32)
    positions = np.stack([[rng.permutation(shape[2]) for _ in range(heads)] for _ in range(2)]).astype(np.int32)
    w, p = torch.from_numpy(weights).cuda(), torch.from_numpy(positions).cuda()
    w_out, p_out, n_out = (w, p, cache.lengths) if in_place else (torch.zeros_like(w), torch.zeros_like(p), torch.zeros_like(cache.lengths))
    work = torch.empty(dq.dq_kv_evict_workspace(2, heads, keep), dtype=torch.uint8, device="cuda")
    dq.dq_kv_evict(cache, w, p, keep, recent, w_out, p_out, n_out, work)
    assert n_out.tolist() == [keep, keep]
    left = kv.Cache(len(c.pages), heads, dim, page, c.table, [keep, keep])
    left.pages = cache.pages.cpu().numpy()
    for b in range(2):
        paged = np.array([c.place(b, slot) is not None for slot in range(length)])
        for h in range(heads):
            source = kv.evict(weights[b, h], positions[b, h], length, keep, recent, paged)
            np.testing.assert_array_equal(p_out[b, h, :keep].cpu().numpy(), positions[b, h, source])
            np.testing.assert_array_equal(w_out[b, h, :keep].cpu().numpy(), weights[b, h, source])
            for slot in np.flatnonzero(paged[:keep]):
                was = int(np.flatnonzero(positions[b, h, :length] == int(p_out[b, h, slot]))[0])
                assert paged[was]
                for second in (0, 1):
                    for one, two in zip(left._at(b, h, slot, second), c._at(b, h, was, second)):
                        assert (one == two).all()
