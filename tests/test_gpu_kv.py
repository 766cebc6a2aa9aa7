"""The operators around the 4-bit key/value cache against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2511_04063_b200 as dq
from kv_util import LEAST, UNIT, attend, check_attention, f64, filled, logit_bound, on_device, put, starts_of, table_of, workspace
from oracle import kv_cache as kv

pytestmark = pytest.mark.gpu

FLOATS = (torch.float32, torch.bfloat16, torch.float16)
HALVES = (torch.bfloat16, torch.float16)


# ------------------------------------------------------------------------------------------------ norm and rotation
def rope_case(tokens, q_heads, k_heads, dim, rot, dtype, flags, seed, views="fused", far=0, gamma_type=None):
    rng = np.random.default_rng(seed)
    heads = q_heads + k_heads
    if views == "fused":                                       # rows of one projection's output
        whole = put(rng.standard_normal((tokens, heads + 3, dim)) * np.exp(rng.standard_normal((tokens, heads + 3, 1))), dtype)
        q, k = whole[:, :q_heads], whole[:, q_heads:heads]
    elif views == "heads first":
        whole = put(rng.standard_normal((heads, tokens, dim)), dtype)
        q, k = whole[:q_heads].transpose(0, 1), whole[q_heads:].transpose(0, 1)
    else:                                                      # heads on no 16-byte boundary
        whole = put(rng.standard_normal((tokens, heads * (dim + 1) + 1)), dtype)
        q = torch.as_strided(whole, (tokens, q_heads, dim), (whole.stride(0), dim + 1, 1), 1)
        k = torch.as_strided(whole, (tokens, k_heads, dim), (whole.stride(0), dim + 1, 1), 1 + q_heads * (dim + 1))
    positions = torch.from_numpy(far + rng.permutation(tokens).astype(np.int32) * 3).cuda().int()
    freq = torch.from_numpy((10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))).astype(np.float32)).cuda() if rot else None
    gamma = [put(1 + 0.2 * rng.standard_normal(dim), gamma_type or dtype) for _ in range(2)] if flags & dq.DQ_QK_NORM else [None, None]
    return q, k, positions, freq, gamma


def check_rope(got, x, positions, freq, gamma, flags, eps=1e-6):
    """All arithmetic is in fp32: a root of a sum of dim squares, products, a pair's sum (and angles to 2^-22), log2(dim) sums of a
    Hadamard rotation; at most 64 roundings of the magnitudes that are summed, then one to the type."""
    dim, dtype = x.shape[-1], x.dtype
    norm = bool(flags & dq.DQ_QK_NORM)
    args = dict(positions=f64(positions), inv_freq=None if freq is None else f64(freq), gamma=None if gamma is None else f64(gamma),
                eps=eps if norm else None, neighbours=bool(flags & dq.DQ_QK_NEIGHBOURS))
    ref = kv.norm_rope(f64(x), **args, hadamard=bool(flags & dq.DQ_QK_HADAMARD))
    plain = np.abs(kv.norm_rope(f64(x), **args))
    if flags & dq.DQ_QK_HADAMARD:
        size = plain.sum(-1, keepdims=True) / np.sqrt(dim)
    else:                                                      # a pair keeps its length
        size = plain.copy()
        for i in range(0 if freq is None else len(freq)):
            a, b = (2 * i, 2 * i + 1) if flags & dq.DQ_QK_NEIGHBOURS else (i, i + len(freq))
            size[..., a] = size[..., b] = plain[..., a] + plain[..., b]
    bound = 64 * 2.0 ** -24 * size * np.sqrt(2) + UNIT[dtype] * np.abs(ref) * 1.01 + LEAST[dtype]
    assert (np.abs(f64(got) - ref) <= bound).all()


def run_rope(q, k, positions, freq, gamma, flags):
    q_out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    k_out = torch.empty(k.shape, dtype=k.dtype, device="cuda")
    dq.dq_qk_norm_rope(q, k, positions, freq, q_out, k_out, q_gamma=gamma[0], k_gamma=gamma[1], flags=flags)
    check_rope(q_out, q, positions, freq, gamma[0], flags)
    check_rope(k_out, k, positions, freq, gamma[1], flags)
    return q_out, k_out


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("dim,rot", [(16, 16), (48, 32), (64, 64), (64, 32), (80, 80), (128, 128), (128, 64), (128, 96), (240, 112), (256, 256), (256, 16)])
@pytest.mark.parametrize("flags", [1, 3, 0])
def test_rope(dtype, dim, rot, flags):
    run_rope(*rope_case(7, 5, 2, dim, rot, dtype, flags, dim + rot), flags)


@pytest.mark.parametrize("dim,rot", [(64, 64), (64, 16), (128, 128), (128, 48), (256, 256), (256, 128), (128, 0)])
@pytest.mark.parametrize("flags", [5, 7, 4])
def test_rope_with_hadamard(dim, rot, flags):
    for dtype in FLOATS:
        run_rope(*rope_case(9, 6, 3, dim, rot, dtype, flags, dim + rot), flags)


@pytest.mark.parametrize("views", ["fused", "heads first", "unaligned"])
@pytest.mark.parametrize("tokens,q_heads,k_heads", [(1, 1, 1), (1, 32, 8), (3, 40, 40), (300, 7, 1), (700, 64, 8)])
def test_rope_sizes_and_views(tokens, q_heads, k_heads, views):
    for dtype, flags in ((torch.bfloat16, 5), (torch.float16, 3), (torch.float32, 1)):
        run_rope(*rope_case(tokens, q_heads, k_heads, 128, 128, dtype, flags, tokens, views), flags)


@pytest.mark.parametrize("tokens,q_heads,k_heads,dim,rot,flags", [(4000, 7, 2, 64, 64, 5), (1500, 10, 3, 128, 128, 5), (4000, 3, 2, 256, 128, 7),
                                                                  (1500, 6, 1, 128, 96, 5), (4000, 5, 1, 80, 64, 1)])
def test_rope_of_many_tokens(tokens, q_heads, k_heads, dim, rot, flags):
    """A warp or a few for each token, which go round over its heads, from queries to keys between two rounds."""
    for views in ("fused", "unaligned"):
        q, k, positions, freq, gamma = rope_case(tokens, q_heads, k_heads, dim, rot, torch.bfloat16, flags, tokens + dim, views)
        run_rope(q, k, positions, freq, gamma, flags)


def test_rope_far_positions_and_gammas():
    q, k, p, f, g = rope_case(5, 3, 1, 128, 128, torch.float32, 1, 3, far=2 ** 31 - 100, gamma_type=torch.float32)
    run_rope(q, k, p, f, g, 1)
    q, k, p, f, g = rope_case(5, 3, 1, 128, 128, torch.bfloat16, 1, 3, far=1000000, gamma_type=torch.float32)
    run_rope(q, k, p, f, g, 1)
    run_rope(q, k, p, f, [None, g[1]], 1)
    run_rope(q, k, -p, f, [None, None], 1)


@pytest.mark.parametrize("flags,rot", [(1, 128), (5, 128), (5, 64), (7, 64)])
def test_rope_in_place_and_without_keys(flags, rot):
    q, k, p, f, g = rope_case(33, 9, 2, 128, rot, torch.bfloat16, flags, 8)
    want_q, want_k = run_rope(q, k, p, f, g, flags)
    only = torch.empty_like(want_q)
    dq.dq_qk_norm_rope(q, None, p, f, only, None, q_gamma=g[0], flags=flags)
    assert torch.equal(only, want_q)
    dq.dq_qk_norm_rope(q, k, p, f, q, k, q_gamma=g[0], k_gamma=g[1], flags=flags)
    assert torch.equal(q, want_q) and torch.equal(k, want_k)


def test_rope_rows_that_are_not_numbers():
    q, k, p, f, g = rope_case(4, 4, 1, 128, 128, torch.float32, 5, 1)
    q = q.clone()
    q[1, 2, 7], q[2, 1] = float("nan"), 0.0
    out = torch.empty_like(q)
    dq.dq_qk_norm_rope(q, None, p, f, out, None, flags=5)
    bad = torch.isnan(out).any(-1)
    assert bool(torch.isnan(out[1, 2]).all()) and int(bad.sum()) == 1 and bool((out[2, 1] == 0).all())


# ------------------------------------------------------------------------------------------------ append and read back
def append_both(rng, queries, lengths, heads, dim, page, dtype, x=None, views=False, more=0):
    """Appends on the device and in the oracle; compares every byte of the pages, the values and the slots' positions."""
    table, n_pages = table_of(rng, lengths, page)
    c = kv.Cache(n_pages, heads, dim, page, table, lengths, 0x5a)
    cache = on_device(c)
    total = sum(queries) + more                                # rows behind the last sequence
    if x is None:
        x = rng.standard_normal((total, 2 * heads, dim)) * np.exp(rng.standard_normal((total, 2 * heads, 1))) + rng.standard_normal(dim)
    both = put(x, dtype)
    if views:
        both = torch.cat((both, both[..., :1]), -1)[..., :dim]    # heads on no 16-byte boundary
    k, v = both[:, :heads], both[:, heads:]
    values = [torch.full((total, heads, dim), 77.0, dtype=dtype, device="cuda") for _ in range(2)]
    positions = torch.arange(1000, 1000 + total, dtype=torch.int32, device="cuda")
    held = torch.full((len(lengths), heads, cache.slots), -7, dtype=torch.int32, device="cuda")
    want_held = held.cpu().numpy()
    dq.dq_kv_append(k, v, cache, starts=starts_of(queries), k_values=values[0], v_values=values[1], positions=positions, slot_positions=held)
    first = 0
    want = [np.full((total, heads, dim), 77.0) for _ in range(2)]
    for b, n in enumerate(queries):
        for i in range(n):
            slot = c.length(b) - n + i
            for h in range(heads):
                for which, t in enumerate((k, v)):
                    row = f64(t[first + i, h])
                    if slot >= 0:
                        want[which][first + i, h] = c.write(b, h, slot, which, row)
                    else:
                        want[which][first + i, h] = kv.value(*kv.quantize(row))
                if slot >= 0:
                    want_held[b, h, slot] = 1000 + first + i
        first += n
    assert (cache.pages.cpu().numpy() == c.pages).all()
    for got, w in zip(values, want):
        assert torch.equal(got, put(w, torch.float64).to(torch.float32).to(dtype)) or \
            np.array_equal(f64(got), f64(put(w, torch.float64).float().to(dtype)), equal_nan=True)
    assert (held.cpu().numpy() == want_held).all()
    back = [torch.full((total, heads, dim), 77.0, dtype=dtype, device="cuda") for _ in range(2)]
    dq.dq_kv_dequantize(cache, back[0], back[1], starts=starts_of(queries))
    first = 0
    for b, n in enumerate(queries):
        lost = max(0, n - c.length(b))                          # tokens without a slot read back as zeros
        for got, w in zip(back, values):
            assert bool((got[first:first + lost] == 0).all())
            assert torch.equal(torch.nan_to_num(got[first + lost:first + n], 123.0), torch.nan_to_num(w[first + lost:first + n], 123.0))
        first += n
    for got in back:
        assert bool((got[first:] == 77).all())


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("dim", (64, 128, 256))
@pytest.mark.parametrize("page", (16, 64))
def test_append(dtype, dim, page):
    rng = np.random.default_rng(dim + page)
    append_both(rng, [1, 5, 0, 33, 20], [1, 40, 17, 33, 130], 3, dim, page, dtype)


def test_append_sizes():
    rng = np.random.default_rng(5)
    append_both(rng, [1], [1], 1, 128, 16, torch.bfloat16)
    append_both(rng, [1] * 40, list(range(1, 41)), 1, 64, 32, torch.float16)
    append_both(rng, [70], [300], 40, 128, 256, torch.bfloat16, views=True)
    append_both(rng, [3, 2], [2, 2], 2, 128, 16, torch.bfloat16, more=4)           # more tokens than slots, rows of nobody


def test_append_values_at_the_quantiser_s_edges():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((24, 2, 128))
    x[0], x[1], x[2] = 0.0, -3.25, 1e-41                      # constants, one of them below fp32's normal numbers
    x[3, :, ::2] = -0.0
    x[3, :, 1::2] = 0.0
    x[4] = np.arange(128) % 16                                # the grid itself, and its ties
    x[5] = (np.arange(128) % 31) / 2
    x[6, :, 0], x[7, :, 1], x[8, :, 2] = np.nan, np.inf, -np.inf
    x[9], x[9, :, 5] = 1000.0, 1000.001                       # a small range far from zero
    x[10, :, :2] = [-3.4e38, 3.4e38]                          # a range past fp32's
    x[11], x[11, :, 3] = 0.0, 3e38
    x[12] *= 1e-39
    for dtype in FLOATS:
        append_both(rng, [24], [24], 1, 128, 16, dtype, x=x)


def test_append_where_the_table_names_no_page():
    rng = np.random.default_rng(7)
    heads, dim, page = 2, 128, 16
    c = kv.Cache(4, heads, dim, page, [[2, -1, 4, 1]], [60], 0)
    cache = on_device(c)
    k, v = (put(rng.standard_normal((60, heads, dim)), torch.bfloat16) for _ in range(2))
    dq.dq_kv_append(k, v, cache)
    for slot in range(60):
        for h in range(heads):
            c.write(0, h, slot, 0, f64(k[slot, h]))
            c.write(0, h, slot, 1, f64(v[slot, h]))
    assert (cache.pages.cpu().numpy() == c.pages).all() and not c.pages[[0, 3]].any()
    back = [torch.full_like(k, 5.0) for _ in range(2)]
    dq.dq_kv_dequantize(cache, *back)
    assert bool((back[0][16:48] == 0).all()) and bool((back[0][:16] != 0).any()) and bool((back[1][48:] != 0).any())


# ------------------------------------------------------------------------------------------------ attention
def attention_case(seed, lengths, queries, heads, group, dim, page, dtype, spread=1.0, q_size=1.0, even=False):
    rng = np.random.default_rng(seed)
    c, cache = filled(rng, lengths, heads, dim, page, spread)
    q = put(q_size * rng.standard_normal((sum(queries), heads * group, dim)), dtype)
    scale = 1 / np.sqrt(dim)
    out, lse = attend(cache, q, scale, None if even else starts_of(queries))
    first = 0
    for b, n in enumerate(queries):
        check_attention(c, b, q, first, n, group, scale, out, lse)
        first += n
    return c, cache, q, out, lse


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 257]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("dim", (64, 128, 256))
@pytest.mark.parametrize("page", (16, 32, 128))
def test_attention_of_one_token_each(dtype, dim, page):
    attention_case(dim, LENGTHS, [1] * len(LENGTHS), 2, 4, dim, page, dtype, even=True)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("dim", (64, 128, 256))
@pytest.mark.parametrize("group,queries", [(1, [1, 7, 16, 3]), (5, [2, 1, 0, 4]), (8, [1, 2, 3, 1]), (16, [1, 1, 1, 2])])
def test_attention_of_a_few_tokens(dtype, dim, group, queries):
    attention_case(group, [70, 33, 40, 5], queries, 2, group, dim, 16, dtype)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("dim", (64, 128, 256))
def test_attention_of_chunks(dtype, dim):
    """Chunks behind a cached prefix, whole prompts, one longer than its cache (its first tokens see nothing)."""
    attention_case(3, [200, 90, 40, 64], [77, 90, 50, 1], 2, 3, dim, 32, dtype)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("dim", (64, 128, 256))
def test_attention_of_chunks_over_a_long_axis(dtype, dim):
    """Many rows of few sequences: a tile's keys are cut between CTAs, with parts that a row sees nothing of."""
    attention_case(5, [1500], [90], 1, 2, dim, 64, dtype)
    attention_case(6, [700, 1030], [300, 20], 2, 1, dim, 16, dtype)


def test_attention_of_chunks_does_not_depend_on_the_run():
    rng = np.random.default_rng(15)
    c, cache = filled(rng, [1300, 90], 2, 128, 64)
    q = put(rng.standard_normal((200, 4, 128)), torch.bfloat16)
    work, starts = workspace(128), starts_of([150, 50])
    first = attend(cache, q, 0.1, starts, work=work)
    check_attention(c, 0, q, 0, 150, 2, 0.1, *first)
    check_attention(c, 1, q, 150, 50, 2, 0.1, *first)
    for _ in range(10):
        again = attend(cache, q, 0.1, starts, work=work)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    few = attend(cache, q[:2], 0.1, starts_of([1, 1]), work=work)      # the other kernels' counters are as they were
    check_attention(c, 0, q, 0, 1, 2, 0.1, *few)
    for scale in (0.0, -0.3):
        out, lse = attend(cache, q, scale, starts, work=work)
        check_attention(c, 1, q, 150, 50, 2, scale, out, lse)
        few = attend(cache, q[150:151], scale, torch.tensor([0, 0, 1], dtype=torch.int32, device="cuda"))
        check_attention(c, 1, q[150:151], 0, 1, 2, scale, *few)


def test_chunks_with_missing_pages_and_values_that_are_not_numbers():
    rng = np.random.default_rng(16)
    for dim in (64, 128, 256):
        c, _ = filled(rng, [300], 1, dim, 16)
        c.table[0, [2, 9, 17]] = -1, len(c.pages), -7
        q = put(rng.standard_normal((100, 2, dim)), torch.float16)
        out, lse = attend(on_device(c), q, 0.1)
        check_attention(c, 0, q, 0, 100, 2, 0.1, out, lse)
        for second in (0, 1):
            bad = kv.Cache(len(c.pages), 1, dim, 16, c.table, [300])
            bad.pages = c.pages.copy()
            bad.write(0, 0, 250, second, np.full(dim, np.nan))          # tokens 200 .. 299: the first 50 do not see it
            out, lse = attend(on_device(bad), q, 0.1)
            seen = kv.Cache(len(c.pages), 1, dim, 16, c.table, [250])
            seen.pages = c.pages
            check_attention(seen, 0, q[:50], 0, 50, 2, 0.1, out[:50], lse[:50])
            assert bool(torch.isnan(out[50:]).all()) and bool(torch.isnan(lse[50:]).all()) == (second == 0)


def test_chunks_over_keys_and_values_of_no_range():
    """Keys and values whose scale is zero (all dimensions the same), of one size or many, alone in a tile of keys and among others."""
    rng = np.random.default_rng(18)
    for dim in (64, 128, 256):
        c, _ = filled(rng, [400], 2, dim, 16)
        for slot in range(400):
            if slot < 270 or slot % 7 == 0:
                for h in range(2):
                    c.write(0, h, slot, 0, np.full(dim, [0.0, -3.25, 1e-3, 2.0][slot % 4] / dim ** 0.5))
                    c.write(0, h, slot, 1, np.full(dim, [0.0, 3.25, -1e4][slot % 3]))
        c.write(0, 1, 5, 0, np.full(dim, 1e20))                       # too large for any query that is not zero
        cache = on_device(c)
        q = rng.standard_normal((130, 4, dim))
        q[:, 2:] = 0.0
        q[129] = 1e-30
        q = put(q, torch.bfloat16)
        for n in (130, 2):                                            # both kernels
            out, lse = attend(cache, q[-n:], 0.1)
            check_attention(c, 0, q[-n:], 0, n, 2, 0.1, out, lse)


def test_chunks_of_views():
    rng = np.random.default_rng(17)
    c, cache = filled(rng, [90], 2, 128, 16)
    whole = put(rng.standard_normal((70, 12, 129)), torch.bfloat16)
    q = whole[:, 2:8, 1:]
    want, lse = attend(cache, q.contiguous(), 0.1)
    check_attention(c, 0, q, 0, 70, 3, 0.1, want, lse)
    out = torch.full((6, 70, 131), 77.0, dtype=torch.bfloat16, device="cuda")
    got, got_lse = attend(cache, q, 0.1, out=out.transpose(0, 1)[..., 1:129])
    assert torch.equal(got, want) and torch.equal(got_lse, lse)
    assert bool((out[..., 0] == 77).all()) and bool((out[..., 129:] == 77).all())


@pytest.mark.parametrize("heads,group,dim", [(1, 1, 64), (1, 8, 128), (2, 2, 256), (8, 4, 128)])
def test_attention_over_a_long_axis(heads, group, dim):
    """Few sequences: the axis is split over all SMs and joined."""
    for n in (1, 3):
        attention_case(n, [2100, 700][:3 - n if n < 3 else 1], [n] * (3 - n if n < 3 else 1), heads, group, dim, 64, torch.bfloat16)


def test_attention_of_many_sequences():
    """More sequences than a CTA has threads; most of them empty or short."""
    lengths = [(7 * i) % 23 for i in range(1200)]
    attention_case(11, lengths, [1] * 1200, 1, 2, 64, 16, torch.float16)


@pytest.mark.parametrize("n_seqs", (40, 600))
def test_chunks_of_many_sequences(n_seqs):
    """More sequences than a warp, and than a CTA, has threads, with 128 rows and more of each on average, some without any."""
    queries = [(0, 17, 18, 16, 33)[i % 5] for i in range(n_seqs)]
    lengths = [n + (i % 4) * 9 if i % 7 else n // 2 for i, n in enumerate(queries)]
    attention_case(12, lengths, queries, 1, 8, 64, 16, torch.bfloat16)


@pytest.mark.parametrize("dtype", HALVES)
def test_attention_with_large_logits(dtype):
    """Logits of some hundreds: one key takes nearly all; and keys far from zero."""
    attention_case(1, [130, 40], [2, 1], 2, 4, 128, 16, dtype, spread=6.0, q_size=8.0)


def test_attention_views():
    rng = np.random.default_rng(2)
    c, cache = filled(rng, [50, 20, 9], 2, 128, 16)
    scale = 0.09
    whole = put(rng.standard_normal((3, 14, 128)), torch.bfloat16)
    q = whole[:, 2:10]
    want, lse = attend(cache, q.contiguous(), scale)
    for b in range(3):
        check_attention(c, b, q, b, 1, 4, scale, want, lse)
    first = put(f64(q), torch.bfloat16).transpose(0, 1).contiguous().transpose(0, 1)
    odd = torch.cat((q, q[..., :1]), -1)[..., :128]
    for view in (q, first, odd):
        out = torch.full((3, 8, 131), 77.0, dtype=torch.bfloat16, device="cuda")
        got, got_lse = attend(cache, view, scale, out=out[..., 2:130])
        assert torch.equal(got, want) and torch.equal(got_lse, lse)
        assert bool((out[..., :2] == 77).all()) and bool((out[..., 130:] == 77).all())
    out = torch.empty_like(want)
    dq.dq_kv_attention(q, cache, scale, out, workspace(128))
    assert torch.equal(out, want)


def test_attention_leaves_rows_of_nobody():
    rng = np.random.default_rng(4)
    c, cache = filled(rng, [50, 20], 2, 64, 16)
    q = put(rng.standard_normal((9, 4, 64)), torch.bfloat16)
    starts = torch.tensor([2, 3, 5], dtype=torch.int32, device="cuda")
    out, lse = attend(cache, q, 0.1, starts)
    check_attention(c, 0, q, 2, 1, 2, 0.1, out, lse)
    check_attention(c, 1, q, 3, 2, 2, 0.1, out, lse)
    for t in (out, lse):
        assert bool((t[:2] == 77).all()) and bool((t[5:] == 77).all())


def test_attention_without_some_pages():
    """Keys without a page take no part; a sequence with none at all is like an empty one; a page named twice counts twice."""
    rng = np.random.default_rng(9)
    for page in (16, 32, 64):
        c, _ = filled(rng, [5 * page + 3, 2 * page, page, 2 * page], 2, 128, page, fill=255)
        c.table[0, [1, 4]] = -1, len(c.pages)
        c.table[1] = -5
        c.table[3, 1] = c.table[3, 0]
        cache = on_device(c)
        q = put(rng.standard_normal((8, 6, 128)), torch.bfloat16)
        out, lse = attend(cache, q, 0.1)
        for b in range(4):
            check_attention(c, b, q, 2 * b, 2, 3, 0.1, out, lse)
        assert bool((out[2:4] == 0).all()) and bool((lse[2:4] == -torch.inf).all())


def test_attention_lengths_out_of_range():
    rng = np.random.default_rng(10)
    c, _ = filled(rng, [64, 64, 0], 2, 64, 16)
    c.lengths[:] = [10 ** 9, 64, -3]                            # taken as the table's width, and as zero
    q = put(rng.standard_normal((3, 2, 64)), torch.float16)
    out, lse = attend(on_device(c), q, 0.1)
    for b in range(3):
        check_attention(c, b, q, b, 1, 1, 0.1, out, lse)


def test_attention_of_values_that_are_not_numbers():
    """A key or value that is NaN reaches the queries that see it, and no others."""
    rng = np.random.default_rng(12)
    for second in (0, 1):
        c, _ = filled(rng, [40], 1, 128, 16)
        c.write(0, 0, 38, second, np.full(128, np.nan))
        q = put(rng.standard_normal((4, 2, 128)), torch.bfloat16)       # tokens 36 .. 39
        out, lse = attend(on_device(c), q, 0.1)
        check_attention(c, 0, q[:2], 0, 0, 2, 0.1, out, lse)
        good = kv.Cache(len(c.pages), 1, 128, 16, c.table, [38])
        good.pages = c.pages
        check_attention(good, 0, q[:2], 0, 2, 2, 0.1, out[:2], lse[:2])
        assert bool(torch.isnan(out[2:]).all())
        assert bool(torch.isnan(lse[2:]).all()) == (second == 0)


def test_attention_does_not_depend_on_the_run_and_leaves_its_workspace_ready():
    rng = np.random.default_rng(13)
    c, cache = filled(rng, [1500, 9, 700], 2, 128, 64)
    q = put(rng.standard_normal((3, 8, 128)), torch.bfloat16)
    work = workspace(128)
    first = attend(cache, q, 0.1, work=work)
    for _ in range(20):
        again = attend(cache, q, 0.1, work=work)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    assert not bool(work[:1024].any())                          # the counters


def test_attention_on_two_streams_and_captured():
    rng = np.random.default_rng(14)
    c, cache = filled(rng, [900, 300], 2, 128, 64)
    q = [put(rng.standard_normal((2, 8, 128)), torch.bfloat16) for _ in range(2)]
    want = [attend(cache, x, 0.1) for x in q]
    streams, works = [torch.cuda.Stream() for _ in range(2)], [workspace(128) for _ in range(2)]
    outs, sums = [torch.zeros_like(x) for x in q], [torch.zeros(x.shape[:2], device="cuda") for x in q]
    torch.cuda.synchronize()
    for _ in range(30):
        for i in range(2):
            dq.dq_kv_attention(q[i], cache, 0.1, outs[i], works[i], lse=sums[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i][0]) and torch.equal(sums[i], want[i][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dq.dq_kv_attention(q[0], cache, 0.1, outs[0], works[0], lse=sums[0])
    cache.lengths.copy_(torch.tensor([401, 300], dtype=torch.int32))   # read when the graph runs
    c.lengths[:] = [401, 300]
    for _ in range(3):
        outs[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for b in range(2):
            check_attention(c, b, q[0], b, 1, 4, 0.1, outs[0], sums[0])


# ------------------------------------------------------------------------------------------------ weights
def weights_case(seed, lengths, queries, heads, group, dim, page, dtype, more=0):
    rng = np.random.default_rng(seed)
    c, cache = filled(rng, lengths, heads, dim, page)
    q = put(rng.standard_normal((sum(queries), heads * group, dim)), dtype)
    scale, starts = 1 / np.sqrt(dim), starts_of(queries)
    _, lse = attend(cache, q, scale, starts)
    shape = (len(lengths), heads, cache.slots + more)
    old = torch.from_numpy(rng.random(shape).astype(np.float32)).cuda()
    out = torch.full(shape, 77.0, device="cuda")
    dq.dq_kv_attention_weights(q, lse, cache, scale, out, weights=old, starts=starts)
    fresh = torch.full(shape, 77.0, device="cuda")
    dq.dq_kv_attention_weights(q, lse, cache, scale, fresh, starts=starts)
    place = old.clone()
    dq.dq_kv_attention_weights(q, lse, cache, scale, place, weights=place, starts=starts)
    first = 0
    for b, n in enumerate(queries):
        length = c.length(b)
        for h in range(heads):
            r = kv.attention(c, b, h, f64(q[first:first + n, h * group:(h + 1) * group]), scale)
            got = r["p"].sum((0, 1))
            # two logits' errors (here and in lse, whose own rounding is counted too), an exponential, a sum of n * group terms
            e = (2 * logit_bound(r["logits"], dim) + 2.0 ** -21 * (2 + np.abs(np.nan_to_num(r["lse"], neginf=0))))[..., None] * r["p"]
            bound = e.sum((0, 1)) + (n * group + 4) * 2.0 ** -24 * got + 2.0 ** -24 + 2.0 ** -30
            assert (np.abs(f64(fresh[b, h, :length]) - got) <= bound).all()
            kept = max(0, length - n)
            want = got + np.where(np.arange(length) < kept, f64(old[b, h, :length]), 0)
            assert (np.abs(f64(out[b, h, :length]) - want) <= bound + 2.0 ** -23 * want).all()
            assert bool((out[b, h, length:] == 77).all()) and bool((fresh[b, h, length:] == 77).all())
            assert torch.equal(place[b, h, :length], out[b, h, :length]) and torch.equal(place[b, h, length:], old[b, h, length:])
        first += n
    return q, lse, cache


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("dim", (64, 128, 256))
def test_weights(dtype, dim):
    weights_case(dim, LENGTHS, [1] * len(LENGTHS), 2, 4, dim, 16, dtype)
    weights_case(dim, [200, 90, 40, 64, 7], [77, 90, 50, 1, 0], 2, 3, dim, 32, dtype, more=5)


def test_weights_of_a_long_axis_and_of_many_sequences():
    weights_case(1, [2100], [2], 2, 8, 128, 64, torch.bfloat16)
    weights_case(2, [(5 * i) % 19 for i in range(600)], [1] * 600, 1, 1, 64, 16, torch.float16)


@pytest.mark.parametrize("n_seqs,n,group", [(40, 3, 8), (600, 3, 8), (34, 66, 8), (3, 70, 16)])
def test_weights_of_chunks_of_many_sequences(n_seqs, n, group):
    """By every number of CTAs that share a block of keys; sequences without queries keep their weights."""
    queries = [0 if i % 9 == 8 else n + i % 3 for i in range(n_seqs)]
    weights_case(3, [q + (i % 5) * 11 for i, q in enumerate(queries)], queries, 1, group, 64, 16, torch.bfloat16)


def test_weights_without_tokens():
    rng = np.random.default_rng(4)
    _, cache = filled(rng, [20, 0, 33], 2, 64, 16)
    old, out = torch.rand((3, 2, cache.slots), device="cuda"), torch.full((3, 2, cache.slots), 77.0, device="cuda")
    dq.dq_kv_attention_weights(torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((0, 4), device="cuda"), cache, 0.1, out,
                               weights=old)
    for b, length in enumerate((20, 0, 33)):
        assert torch.equal(out[b, :, :length], old[b, :, :length]) and bool((out[b, :, length:] == 77).all())


# ------------------------------------------------------------------------------------------------ eviction
def evict_case(rng, lengths, heads, dim, page, keep, recent, weights=None, positions=None, in_place=False, missing=False):
    c, _ = filled(rng, lengths, heads, dim, page)
    if missing:
        c.table[0, 0] = -1
    cache = on_device(c)
    shape = (len(lengths), heads, cache.slots + 3)
    if weights is None:
        weights = rng.exponential(size=shape).astype(np.float32)
    if positions is None:
        positions = np.stack([[rng.permutation(shape[2]) for _ in range(heads)] for _ in lengths]).astype(np.int32)
    w, p = torch.from_numpy(weights).cuda(), torch.from_numpy(positions).cuda()
    if in_place:
        w_out, p_out, n_out = w, p, cache.lengths
    else:
        w_out, p_out, n_out = torch.full_like(w, 77.0), torch.full_like(p, 77), torch.zeros_like(cache.lengths)
    before_w, before_p = w_out.cpu().numpy().copy(), p_out.cpu().numpy().copy()
    work = torch.full((dq.dq_kv_evict_workspace(len(lengths), heads, keep),), 255, dtype=torch.uint8, device="cuda")
    dq.dq_kv_evict(cache, w, p, keep, recent, w_out, p_out, n_out, work)
    pages = c.pages.copy()
    for b in range(len(lengths)):
        n = c.length(b)
        for h in range(heads):
            source = kv.evict(weights[b, h], positions[b, h], n, keep, recent)
            before_w[b, h, :len(source)], before_p[b, h, :len(source)] = weights[b, h, source], positions[b, h, source]
            for to, at in enumerate(source):
                if to == at:
                    continue
                for second in (0, 1):
                    one, two = c._at(b, h, at, second), c._at(b, h, to, second)
                    if one is None or two is None:
                        continue
                    page, group, t = c.place(b, to)
                    base = group + second * 16 * (dim // 2 + 4)
                    pages[page, h, base + t * dim // 2:base + (t + 1) * dim // 2] = one[0]
                    pages[page, h, base + 8 * dim + 4 * t:base + 8 * dim + 4 * t + 4] = one[1]
    np.testing.assert_array_equal(p_out.cpu().numpy(), before_p)
    np.testing.assert_array_equal(w_out.cpu().numpy(), before_w)
    assert n_out.cpu().tolist() == [min(c_len, keep) for c_len in (c.length(b) for b in range(len(lengths)))]
    assert (cache.pages.cpu().numpy() == pages).all()


@pytest.mark.parametrize("dim", (64, 128, 256))
@pytest.mark.parametrize("in_place", (False, True))
def test_evict(dim, in_place):
    rng = np.random.default_rng(dim)
    evict_case(rng, [0, 1, 40, 41, 57, 130], 2, dim, 16, 40, 8, in_place=in_place)
    evict_case(rng, [33, 20], 3, dim, 32, 1, 1, in_place=in_place)
    evict_case(rng, [33, 20], 3, dim, 32, 1, 0, in_place=in_place)


def test_evict_long_rows_ties_and_odd_weights():
    rng = np.random.default_rng(1)
    evict_case(rng, [2600], 1, 64, 64, 1030, 100)
    shape = (2, 2, 256 + 3)
    few = rng.integers(0, 3, shape).astype(np.float32)           # many equals: the lower slots stay
    evict_case(rng, [250, 200], 2, 64, 16, 100, 10, weights=few)
    odd = rng.standard_normal(shape).astype(np.float32)
    odd[..., ::7], odd[..., 1::7], odd[..., 2::7] = np.nan, -0.0, 0.0
    odd[..., 3::70], odd[..., 4::70] = np.inf, -np.inf
    evict_case(rng, [250, 200], 2, 64, 16, 120, 0, weights=odd)
    evict_case(rng, [250, 200], 2, 64, 16, 220, 0, weights=odd)
    evict_case(rng, [250, 200], 2, 64, 16, 100, 100)             # all of them recent ones
    same = np.zeros(shape, np.int32)                             # more protected ones than may stay
    evict_case(rng, [250, 200], 2, 64, 16, 100, 5, positions=same)
    far = np.stack([[rng.permutation(259) + 2 ** 31 - 300 for _ in range(2)] for _ in range(2)]).astype(np.int32)
    evict_case(rng, [250, 200], 2, 64, 16, 100, 30, positions=far)
    evict_case(rng, [250, 200], 2, 64, 16, 100, 30, positions=-far)
    evict_case(rng, [60, 50], 2, 64, 16, 20, 3, missing=True)


def test_evict_rows_of_several_blocks():
    """More slots than a CTA holds keys of (weights and positions alone: the cache has no pages)."""
    rng = np.random.default_rng(2)
    lengths, heads, page, keep = [70001, 32768, 32769], 2, 4096, 20000
    table = np.full((3, 18), -1)
    cache = on_device(kv.Cache(1, heads, 64, page, table, lengths))
    shape = (3, heads, cache.slots)
    weights = rng.integers(0, 5000, shape).astype(np.float32)
    positions = np.stack([[rng.permutation(shape[2]) for _ in range(heads)] for _ in lengths]).astype(np.int32)
    w, p = torch.from_numpy(weights).cuda(), torch.from_numpy(positions).cuda()
    w_out, p_out, n_out = torch.zeros_like(w), torch.zeros_like(p), torch.zeros_like(cache.lengths)
    work = torch.empty(dq.dq_kv_evict_workspace(3, heads, keep), dtype=torch.uint8, device="cuda")
    dq.dq_kv_evict(cache, w, p, keep, 100, w_out, p_out, n_out, work)
    assert n_out.tolist() == [keep] * 3
    for b, n in enumerate(lengths):
        for h in range(heads):
            source = kv.evict(weights[b, h], positions[b, h], n, keep, 100)
            np.testing.assert_array_equal(p_out[b, h, :keep].cpu().numpy(), positions[b, h, source])
            np.testing.assert_array_equal(w_out[b, h, :keep].cpu().numpy(), weights[b, h, source])


# ------------------------------------------------------------------------------------------------ together
def test_a_decoding_loop():
    """Prompts, then tokens one by one: norm and rotation, append, attention, weights, eviction, against the oracle's cache that is
    read back from the device after each step."""
    rng = np.random.default_rng(21)
    heads, group, dim, page, keep, recent = 2, 4, 128, 16, 48, 12
    prompts = [30, 50]
    table, n_pages = table_of(rng, [96, 96], page)
    c = kv.Cache(n_pages, heads, dim, page, table, [0, 0], 255)
    cache = on_device(c)
    weights = torch.zeros((2, heads, cache.slots), device="cuda")
    held = torch.full((2, heads, cache.slots), -1, dtype=torch.int32, device="cuda")
    freq = torch.from_numpy((10000.0 ** (-np.arange(dim // 2) / (dim // 2))).astype(np.float32)).cuda()
    work, evict_work = workspace(dim), torch.empty(dq.dq_kv_evict_workspace(2, heads, keep), dtype=torch.uint8, device="cuda")
    scale, seen = 1 / np.sqrt(dim), [0, 0]
    for step in range(20):
        n = prompts if step == 0 else [1, 1]
        x = put(rng.standard_normal((sum(n), (group + 2) * heads, dim)), torch.bfloat16)
        q, k, v = x[:, :group * heads], x[:, group * heads:-heads], x[:, -heads:]
        positions = torch.cat([torch.arange(seen[b], seen[b] + n[b]) for b in range(2)]).int().cuda()
        dq.dq_qk_norm_rope(q, k, positions, freq, q, k, flags=dq.DQ_QK_NORM | dq.DQ_QK_HADAMARD)
        cache.lengths.add_(torch.tensor(n, dtype=torch.int32, device="cuda"))
        starts = starts_of(n)
        dq.dq_kv_append(k, v, cache, starts=starts, positions=positions, slot_positions=held)
        out, lse = attend(cache, q, scale, starts, work=work)
        old = weights.clone()
        dq.dq_kv_attention_weights(q, lse, cache, scale, weights, weights=weights, starts=starts)
        c.pages, c.lengths = cache.pages.cpu().numpy(), cache.lengths.cpu().numpy().astype(np.int64)
        first = 0
        for b in range(2):
            check_attention(c, b, q, first, n[b], group, scale, out, lse)
            for h in range(heads):
                r = kv.attention(c, b, h, f64(q[first:first + n[b], h * group:(h + 1) * group]), scale)
                length = c.length(b)
                want = r["p"].sum((0, 1)) + np.where(np.arange(length) < length - n[b], f64(old[b, h, :length]), 0)
                assert np.abs(f64(weights[b, h, :length]) - want).max() <= 1e-4 * max(1, want.max())
                kept = held[b, h, :length].cpu().numpy()
                assert len(set(kept)) == length and kept.max() == seen[b] + n[b] - 1 and kept.min() >= 0
            first += n[b]
            seen[b] += n[b]
        dq.dq_kv_evict(cache, weights, held, keep, recent, weights, held, cache.lengths, evict_work)
        assert cache.lengths.tolist() == [min(length, keep) for length in c.lengths]
        for b in range(2):
            for h in range(heads):
                kept = set(held[b, h, :int(cache.lengths[b])].tolist())
                assert set(range(seen[b] - recent, seen[b])) <= kept


@pytest.mark.parametrize("tokens", (1, 40))
def test_the_operators_captured_together(tokens):
    """A step of all operators replayed, as it runs by itself on the current stream and on another: the same bytes."""
    rng = np.random.default_rng(22)
    heads, group, dim, page, keep, n_seqs = 2, 4, 128, 16, 96, 3
    table, n_pages = table_of(rng, [keep + 2 * tokens] * n_seqs, page)
    x = [put(rng.standard_normal((n_seqs * tokens, (group + 2) * heads, dim)), torch.bfloat16) for _ in range(6)]
    freq = torch.from_numpy((10000.0 ** (-np.arange(dim // 2) / (dim // 2))).astype(np.float32)).cuda()

    class State:
        def __init__(self):
            self.cache = on_device(kv.Cache(n_pages, heads, dim, page, table, [0] * n_seqs, 0))
            self.x = torch.empty_like(x[0])
            self.positions = (torch.arange(tokens, dtype=torch.int32).repeat(n_seqs) - tokens).cuda()
            self.weights = torch.zeros((n_seqs, heads, self.cache.slots), device="cuda")
            self.held = torch.zeros((n_seqs, heads, self.cache.slots), dtype=torch.int32, device="cuda")
            self.out = torch.empty_like(x[0][:, :group * heads])
            self.lse = torch.empty((n_seqs * tokens, group * heads), device="cuda")
            self.work, self.evict_work = workspace(dim), torch.empty(dq.dq_kv_evict_workspace(n_seqs, heads, keep), dtype=torch.uint8, device="cuda")

        def step(self, stream=None):
            q, k, v = self.x[:, :group * heads], self.x[:, group * heads:-heads], self.x[:, -heads:]
            self.positions.add_(tokens)
            self.cache.lengths.add_(tokens)
            dq.dq_qk_norm_rope(q, k, self.positions, freq, q, k, flags=dq.DQ_QK_NORM | dq.DQ_QK_HADAMARD, stream=stream)
            dq.dq_kv_append(k, v, self.cache, positions=self.positions, slot_positions=self.held, stream=stream)
            dq.dq_kv_attention(q, self.cache, 0.1, self.out, self.work, lse=self.lse, stream=stream)
            dq.dq_kv_attention_weights(q, self.lse, self.cache, 0.1, self.weights, weights=self.weights, stream=stream)
            dq.dq_kv_evict(self.cache, self.weights, self.held, keep, 8, self.weights, self.held, self.cache.lengths, self.evict_work, stream=stream)

        def all(self):
            return [self.cache.pages, self.cache.lengths, self.weights, self.held, self.out, self.lse]

    eager, other, replayed = State(), State(), State()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        replayed.step()
    for data in x * (4 if tokens > 1 else 20):
        eager.x.copy_(data)
        eager.step()
        with torch.cuda.stream(side):
            other.x.copy_(data)
            other.step(side)
        replayed.x.copy_(data)
        graph.replay()
    torch.cuda.synchronize()
    assert eager.cache.lengths.tolist() == [keep] * n_seqs
    for one, two, three in zip(eager.all(), other.all(), replayed.all()):
        assert torch.equal(one, two) and torch.equal(one, three)
    assert dq.dq_mx_status() == dq.DQ_OK and dq.dq_mx_status(side) == dq.DQ_OK
