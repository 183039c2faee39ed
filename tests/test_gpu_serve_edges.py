"""The 8-bit serving operators where they can go wrong: outputs wider than one pass of a kernel, refused calls and what comes behind
them, values of very different sizes, numbers out of range.  Helpers, oracle and the way tolerances are counted: test_gpu_serve.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from test_gpu_serve import ACTS, DTYPES, U, attention_bound, code_weights, ctx, dev, half_step, host, ints, linear_bound, make, same_cache, same_pool, starts_of, steps  # noqa: F401
from test_gpu_serve import test_linear as linear_against_oracle

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- linear layers wider than one pass of a block

@pytest.mark.parametrize("m,k,n", [(1, 100, 50257), (1, 2304, 19001), (8, 100, 32001), (8, 777, 50257), (8, 2304, 19001), (9, 777, 32001), (16, 100, 50257),
                                   (16, 2304, 19001), (16, 4097, 38000)])
@pytest.mark.parametrize("dtype,act,with_bias", [(torch.float32, "none", False), (torch.bfloat16, "relu", True)])
def test_linear_of_few_tokens_into_many_columns(ctx, m, k, n, dtype, act, with_bias):
    """More than eight tiles of 16 columns for each SM: two and three passes of a block, the last one short, with numbers of runs that leave
    warps without one and take the ring of stages through all its places."""
    linear_against_oracle(ctx, m, k, n, dtype, act, with_bias)


def test_linear_of_few_tokens_into_many_strided_columns(ctx):
    rng = np.random.default_rng(3)
    m, k, n = 5, 300, 40003
    x = dev(rng.standard_normal((m, k)).astype(np.float32), torch.float16)
    w, sw = code_weights(rng, n, 304)
    w[:, k:] = 0
    room = torch.full((m + 2, n + 9), 7.0, dtype=torch.float16, device="cuda")
    ctx.linear_i8(x, w, sw, out=room[1:m + 1, 3:3 + n])
    qx, sx = so.quantize_tokens(host(x))
    want, tol = linear_bound(qx, sx, host(w)[:, :k], host(sw), None, "none", torch.float16)
    assert (np.abs(host(room[1:m + 1, 3:3 + n]) - want) <= tol).all()
    room[1:m + 1, 3:3 + n] = 7
    assert (room == 7).all()
    ctx.check_sync()


# ----------------------------------------------------------------------------- what surfaces

def test_every_cause_surfaces(ctx):
    """A value that is not finite does not hide pages that ran out, and the other way round: one cause a call, the gravest first."""
    import paper_2302_01382_b200 as q
    pool, cache, po, co = make(ctx, 4, 16, 2, 4)
    x = torch.full((3, 8), float("nan"), device="cuda")
    for order in (0, 1):
        if order:
            ctx.quantize_tokens(x)
        pool.extend(ints([0]), ints([0, 65]))          # longer than a row of the table
        ctx.quantize_tokens(x)
        assert [ctx.sync_status() for _ in range(4)] == [q.EPAGE, q.ENONFINITE, q.OK, q.OK]
    ctx.quantize_tokens(x)
    ctx.selftest_wait_timeout(1000)
    pool.free(ints([2]))
    assert [ctx.sync_status() for _ in range(4)] == [q.ETIMEOUT, q.EPAGE, q.ENONFINITE, q.OK]
    side = torch.cuda.Stream()
    pool.free(ints([2]), stream=side)
    assert ctx.sync_status(side) == q.EPAGE
    ctx.check_sync()
    same_pool(pool, po)


# ----------------------------------------------------------------------------- no room

def contents(cache):
    return [t.clone() for t in (cache.k, cache.v, cache.k_absmax, cache.v_absmax)]


def unchanged(before, cache):
    return all(torch.equal(a, b) for a, b in zip(before, contents(cache)))


@pytest.mark.parametrize("captured", [False, True])
def test_append_behind_a_refused_extend_writes_nothing(ctx, captured):
    """extend, append without a look at the status in between: with too few pages the last tokens stay, and the step can be repeated."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(31)
    pool, cache, po, co = make(ctx, 6, 16, 4, 4)
    steps(ctx, pool, cache, po, co, [0, 1, 2], [32, 20, 16], torch.float32, rng)       # 5 of 6 pages
    before = contents(cache)
    seqs, shape = [0, 1, 2], (3, 2, 64)
    k, v = (dev(50 * rng.standard_normal(shape).astype(np.float32)) for _ in range(2))
    sd = ints(seqs)

    def step():
        pool.extend(sd)                            # two more pages: one too many
        cache.append(k, v, sd)

    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        step = graph.replay
    for _ in range(2):
        step()
        assert ctx.sync_status() == q.EPAGE and ctx.sync_status() == q.OK
        assert unchanged(before, cache)
        same_pool(pool, po)
    # others go on meanwhile; a refused one stays out until it gets its room
    pool.extend(ints([1]))
    cache.append(k[1:2], v[1:2], ints([1]))
    ctx.check_sync()
    assert po.extend([1], [1])
    co.append(host(k)[1:2], host(v)[1:2], [1], [0, 1])
    same_cache(cache, co)
    cache.append(k[:1], v[:1], ints([0]))
    assert ctx.sync_status() == q.EPAGE
    same_cache(cache, co)
    pool.free(ints([1]))
    po.free([1])
    step()
    ctx.check_sync()
    assert po.extend(seqs, [1, 1, 1])
    co.append(host(k), host(v), seqs, [0, 1, 2, 3])
    same_pool(pool, po)
    same_cache(cache, co)


def test_room_of_other_calls_and_of_sequences_that_begin_again(ctx):
    """A refused call keeps its own sequences out and no others; two calls may make the room of one append; a sequence that was given
    back or forked begins anew."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(37)
    pool, cache, po, co = make(ctx, 8, 16, 5, 3)
    steps(ctx, pool, cache, po, co, [0, 1], [40, 10], torch.float32, rng)
    x = rng.standard_normal((9, 2, 64)).astype(np.float32)
    before = contents(cache)
    pool.extend(ints([0, 2]), ints([0, 9, 9]))     # longer than a row of the table
    pool.extend(ints([1]), ints([0, 4]))
    pool.extend(ints([1]), ints([0, 5]))
    cache.append(dev(x), dev(x), ints([0]), ints([0, 9]))
    assert ctx.sync_status() == q.EPAGE
    assert unchanged(before, cache) and pool.refused.tolist() == [1, 0, 1, 0, 0]
    cache.append(dev(x), dev(x), ints([1]), ints([0, 9]))
    assert po.extend([1], [4]) and po.extend([1], [5])
    co.append(x, x, [1], [0, 9])
    same_pool(pool, po)
    same_cache(cache, co)
    for twice in ([1, 1], [1, 5]):
        pool.extend(ints(twice))
        assert ctx.sync_status() == q.EPAGE and pool.refused.tolist() == [1, 1, 1, 0, 0]
    pool.free(ints([0]))
    po.free([0])
    src, dst = pool.fork(ints([1]), ints([2]))
    cache.copy_pages(src, dst)
    co.copy_pages(*po.fork([1], [2]))
    assert pool.refused.tolist() == [0, 1, 0, 0, 0]
    steps(ctx, pool, cache, po, co, [2, 0, 1], [3, 4, 2], torch.float32, rng)
    ctx.check_sync()
    assert not pool.refused.any()
    same_pool(pool, po)
    same_cache(cache, co)
    pool._c.refused_dev = None
    with pytest.raises(q.QcfgError) as e:
        pool.extend(ints([0]))
    assert e.value.status == q.EINVAL


# ----------------------------------------------------------------------------- digits of the weights

def lone_score(ctx, score, length, rows, heads, dtype, **kw):
    """`length` tokens with values of 1, whose weights are all the same, next to one with a value of 0 whose score is `score` above theirs.
    Returns the output and its exact value: errors of the many weights do not cancel."""
    import paper_2302_01382_b200 as q
    dim, page = 64, 64
    pool = q.KvPool(ctx, -(-length // page) + 1, page, 1, -(-length // page) + 1)
    cache = q.KvCache(pool, heads, dim)
    k = torch.zeros((length, heads, dim), device="cuda")
    v = torch.ones((length, heads, dim), device="cuda")
    at = length // 3
    k[at, :, 5], v[at] = 1.0, 0.0
    seqs, st = ints([0]), ints([0, length])
    pool.extend(seqs, st)
    cache.append(k, v, seqs, st)
    x = torch.zeros((rows, heads, dim), device="cuda")
    x[:, :, 5] = score
    out = cache.attention(x.to(dtype), seqs, ints([0, rows]), sm_scale=1.0, causal=False, **kw)
    ctx.check_sync()
    scale = np.float64(so.scales(np.float32(1))[0]) * 127
    s = host(x.to(dtype))[0, 0, 5].astype(np.float64) * scale
    rest = (length - 1) * np.exp(-s)
    return host(out), scale * rest / (1 + rest), rest, s


@pytest.mark.parametrize("score", [6.5, 9.2, 11.0, 12.7, 14.9])
@pytest.mark.parametrize("rows,heads,max_len", [(1, 2, 0), (12, 2, 0), (1, 2, 512), (12, 2, 512), (300, 26, 0)])
def test_fp32_weights_keep_their_digits_in_the_tail(ctx, score, rows, heads, max_len):
    """The score: fp32 queries to 2^-22, three scalings; the exponential and its argument (up to 22 binary orders) 2^-20; a weight 2^-22, and
    what lies below the fp16 grid 2^-34 of the largest.  Sums of positive numbers, each addition off by U or, in a tensor core, which cuts,
    2 U, and a product of 16 tokens is 16 additions.  A few rows stream over parts of up to 320 tokens by four warps: two halves of 80
    tokens, 10 additions of weights and some 20 parts, below 400 U; a context that is not cut (the hint says it is short) gives a warp
    length / 4 tokens, two halves each, and an addition of weights for each 8.  A block that takes many rows walks the whole context, an
    addition for each token and length / 128 + 30 of weights."""
    length = 40000
    out, want, rest, s = lone_score(ctx, score, length, rows, heads, torch.float32, max_new=rows, max_len=max_len)
    adds = 2 * length + length / 128 + 30 if rows > 32 else 400 + (length / 4 * (4 + 1 / 8) if max_len else 0)
    d_score = s * (2.0 ** -22 + 6 * U) + 2.0 ** -20
    tol = want * (d_score / (1 + rest) + 2.0 ** -22 + adds * U) + length * 2.0 ** -34 / (1 + rest) + U
    assert (np.abs(out - want) <= tol).all(), (float(np.abs(out - want).max()), tol)


def seen_bound(q, k, v, page, sm_scale, causal, window, dtype):
    """Oracle and |error| with nothing in it but the tokens a row sees.  As attention_bound, with this for weights below the fp16 grid: a
    product of weight and page scale is off by 2^-25 where the row's largest is 2^5 or more (in fp32 calls 2^-25 next to 2^8 where all are held
    times 2^9, 2^-35 next to 2^2 where the second halves are held times 2^10 besides); codes are at most 127 of a page's scale, and the weights of all tokens add up."""
    rows, q_heads, dim = q.shape
    length, heads, _ = k.shape
    out, weight, spread = so.attention(q, k, v, sm_scale, causal, window)
    mask = so.seen(rows, length, causal, window)
    pages = np.arange(length) // page
    tops = np.stack([np.abs(v[pages == j]).max((0, 2)) for j in range(pages[-1] + 1)])[pages]      # [length, heads]: at most the page's maximum
    tol = np.zeros(q.shape)
    for h in range(q_heads):
        kh, top = k[:, h // (q_heads // heads)], tops[:, h // (q_heads // heads)]
        s = np.where(mask, q[:, h].astype(np.float64) @ kh.T * sm_scale, -np.inf)
        some = mask.any(1)
        p = np.where(mask, np.exp(s - np.where(some, s.max(1), 0)[:, None]), 0)
        p /= np.where(some, p.sum(1), 1)[:, None]
        largest = (p * top[None, :]).max(1)
        # the largest element of the keys a row sees, times the query's: what queries of 16 bits in fp16 lose
        biggest = np.abs(q[:, h]).max(1) * np.where(mask, np.abs(kh).sum(1)[None, :], 0).max(1) * sm_scale
        score = (dim + 6) * U * spread[:, h] + 2.0 ** -22 * (spread[:, h] + biggest) + 2.0 ** -21
        rel = 2 * np.expm1(score) + (2.0 ** -11 if dtype != torch.float32 else 2.0 ** -20) + (length + 8) * U
        tol[:, h] = rel[:, None] * weight[:, h] + (mask.sum(1) * largest * 2.0 ** (-30 if dtype != torch.float32 else -33))[:, None]
    return out, tol + half_step(dtype) * np.abs(out) + (2.0 ** -25 if dtype == torch.float16 else 1e-38)


@pytest.mark.parametrize("size", [2.0 ** 10, 1e6, 1e12, 1e30])
@pytest.mark.parametrize("page,q_heads,heads,dim", [(16, 4, 2, 64), (32, 8, 1, 128), (16, 3, 3, 80), (64, 26, 26, 64), (16, 32, 8, 128)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_row_does_not_depend_on_values_it_does_not_see(ctx, dtype, page, q_heads, heads, dim, size):
    """Values far larger than the others come later (causal rows in front of them) and came earlier (a window has left them): to a row that
    does not see them they are nothing, though it shares tiles with rows that do."""
    rng = np.random.default_rng(page + dim)
    pool, cache, po, co = make(ctx, 600 // page + 8, page, 2, 512 // page + 2, heads, dim)
    one = torch.float32
    steps(ctx, pool, cache, po, co, [0], [2 * page], one, rng, spread=size)
    steps(ctx, pool, cache, po, co, [0], [256 - 2 * page], one, rng)
    steps(ctx, pool, cache, po, co, [0], [11], one, rng, spread=size)
    # one whose first page is as the others
    steps(ctx, pool, cache, po, co, [1], [256 - page], one, rng)
    steps(ctx, pool, cache, po, co, [1], [9], one, rng, spread=size)
    # the keys stay as they are: their size is not the question here
    cache.k_absmax.clamp_(max=4.0)
    co.absmax[0] = np.minimum(co.absmax[0], np.float32(4))
    ctx.check_sync()
    for seqs, rows, kw in (([1], [12], {}), ([1], [20], {"max_len": 300}), ([1], [po.lens[1]], {"max_new": po.lens[1]}), ([0], [40], {"window": 100}),
                           ([0], [po.lens[0]], {"window": 3 * page + 5, "max_new": po.lens[0]}), ([0, 1], [267, 249 - page], {"max_new": 267, "window": 24})):
        x = dev((rng.standard_normal((sum(rows), q_heads, dim))).astype(np.float32), dtype)
        got = host(cache.attention(x, ints(seqs), ints(starts_of(rows)), **kw))
        at = 0
        for s, c in zip(seqs, rows):
            k, v = co.values(s)
            want, tol = seen_bound(host(x)[at:at + c], k, v, page, dim ** -0.5, True, kw.get("window", 0), dtype)
            ok = np.abs(want) + tol < torch.finfo(dtype).max         # (what the bound lets pass the type's end may be Inf)
            worst = np.where(ok, np.abs(got[at:at + c] - want) - tol, 0)
            assert (worst <= 0).all(), (s, c, kw, float(worst.max()), np.argwhere(worst > 0)[:4].tolist(), len(np.argwhere(worst > 0)))
            at += c
    ctx.check_sync()


@pytest.mark.parametrize("small,large", [(1e-25, 1e20), (1e-4, 1e35), (1e-36, 1.0)])
@pytest.mark.parametrize("page,q_heads,heads,dim", [(16, 4, 2, 64), (32, 8, 1, 128), (16, 3, 3, 80), (64, 26, 26, 64), (16, 32, 8, 128)])
@pytest.mark.parametrize("dtype", DTYPES[:2])
def test_rows_of_a_tile_that_see_values_of_any_size(ctx, dtype, page, q_heads, heads, dim, small, large):
    """Rows that see small values only share tiles with rows that see large ones, up to 2^150 apart, further than the factors of one row's
    may be from another's in fp32.  A weight below 2^-125 of the largest may be 0."""
    rng = np.random.default_rng(page + dim)
    pool, cache, po, co = make(ctx, 300 // page + 8, page, 1, 300 // page + 2, heads, dim)
    for n, size in ((100 // page * page + page, small), (9, large), (13, small)):
        steps(ctx, pool, cache, po, co, [0], [n], torch.float32, rng, spread=size)
    cache.k_absmax.fill_(4.0)                      # keys of ordinary size
    co.absmax[0][:] = 4
    length = po.lens[0]
    k, v = co.values(0)
    for rows, kw in ((30, {}), (30, {"window": 20}), (30, {"max_len": 200}), (length, {"max_new": 400}), (length, {"max_new": 400, "window": 20})):
        x = dev(rng.standard_normal((rows, q_heads, dim)).astype(np.float32), dtype)
        got = host(cache.attention(x, ints([0]), ints([0, rows]), **kw))
        want, tol = seen_bound(host(x), k, v, page, dim ** -0.5, True, kw.get("window", 0), dtype)
        mask = so.seen(rows, length, True, kw.get("window", 0))
        for h in range(q_heads):
            tol[:, h] += 2.0 ** -125 * np.where(mask, np.abs(v[:, h // (q_heads // heads)]).max(1)[None, :], 0).sum(1)[:, None]
        worst = np.abs(got - want) - tol
        assert (worst <= 0).all(), (rows, kw, float(worst.max()), np.argwhere(worst > 0)[:4].tolist(), len(np.argwhere(worst > 0)))
    ctx.check_sync()


# ----------------------------------------------------------------------------- rows out of range

@pytest.mark.parametrize("starts", [[0, 2, 7], [0, 2, 1], [-1, 2, 4], [0, 2, -3]])
def test_entries_whose_rows_are_not_there_are_left_out(ctx, starts):
    """Rows behind the tensors' end, before their begin, or that end before they begin: reported, not cut to what is there; the entry
    beside them is served (but for extend, which is all or nothing)."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(43)
    for dtype, heads, many in ((torch.float32, 2, 1), (torch.bfloat16, 2, 1), (torch.float16, 26, 100)):
        pool, cache, po, co = make(ctx, 40, 16, 3, 16, heads, 64)
        steps(ctx, pool, cache, po, co, [0, 1], [20 * many % 240, 37], torch.float32, rng)
        good, bad = [], []
        for i in range(2):
            lo, hi = starts[i], starts[i + 1]
            (good if 0 <= lo <= hi <= 4 else bad).append(i)
        assert bad
        st, n = ints([s * many for s in starts]), 4 * many
        before = contents(cache)
        pool.extend(ints([0, 1]), st, rows=n)
        assert ctx.sync_status() == q.EPAGE
        same_pool(pool, po)
        pool.refused.zero_()
        x = dev(rng.standard_normal((n, heads, 64)).astype(np.float32), dtype)
        out = torch.full((n, heads, 64), 9.0, dtype=dtype, device="cuda")
        cache.attention(x, ints([0, 1]), st, out=out, max_new=many * 2)
        assert ctx.sync_status() == q.EPAGE
        for i in good:
            rows = slice(many * starts[i], many * starts[i + 1])
            want, tol = attention_bound(host(x[rows]), *co.values(i), 64 ** -0.5, True, 0, dtype)
            assert (np.abs(host(out[rows]) - want) <= tol).all()
            out[rows] = 9
        assert (out == 9).all()                        # nobody's rows are not written
        if many == 1:
            cache.append(x, x, ints([0, 1]), st)
            assert ctx.sync_status() == q.EPAGE
            for i in bad:
                for a, b in zip(before, contents(cache)):
                    for page in po.table[i]:
                        assert torch.equal(a[page], b[page])
        k, v = cache.read(ints([0, 1]), ints([0, 0]), st, n)
        assert ctx.sync_status() == q.EPAGE


# ----------------------------------------------------------------------------- strides nobody uses

@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_of_one_row_or_one_head_do_not_matter(ctx, dtype):
    """A single row of a matrix of odd width, a single head between others, keys and values that differ in such a stride only."""
    rng = np.random.default_rng(47)
    for heads, rows in ((2, 1), (1, 3), (1, 1)):
        pool, cache, po, co = make(ctx, 8, 16, 2, 4, heads, 64)
        steps(ctx, pool, cache, po, co, [0], [20], dtype, rng)
        x = dev(rng.standard_normal((rows, heads, 64)).astype(np.float32), dtype)
        odd = torch.empty_strided(x.shape, (heads * 64 + 5 if rows == 1 else 72 * heads, 67 if heads == 1 else 64, 1), dtype=dtype, device="cuda")
        odd.copy_(x)
        seqs, st = ints([0]), ints([0, rows])
        pool.extend(seqs, st)
        assert po.extend([0], [rows])
        cache.append(odd, odd if rows > 1 else x, seqs, st)
        co.append(host(x), host(x), [0], [0, rows])
        same_cache(cache, co)
        want = cache.attention(x, seqs, st)
        out = torch.empty_strided(x.shape, odd.stride(), dtype=dtype, device="cuda")
        assert torch.equal(cache.attention(odd, seqs, st, out=out), want)
        ctx.check_sync()
    w, s = code_weights(rng, 1, 64)
    out = torch.empty_strided((3, 1), (4, 7), dtype=dtype, device="cuda")
    x = dev(rng.standard_normal((3, 64)).astype(np.float32), dtype)
    assert torch.equal(ctx.linear_i8(x, w, s, out=out), ctx.linear_i8(x, w, s))


def test_a_type_that_is_not_the_outputs_is_refused(ctx):
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(53)
    x = dev(rng.standard_normal((5, 64)).astype(np.float32), torch.bfloat16)
    w, s = code_weights(rng, 32, 64)
    codes, sx = ctx.quantize_tokens(x)
    for call in (lambda **kw: ctx.linear_i8(x, w, s, **kw), lambda **kw: ctx.gemm_i8_token(codes, w, 64, sx, s, **kw)):
        out = torch.zeros((5, 32), dtype=torch.float16, device="cuda")
        for other in (torch.float32, torch.bfloat16):
            with pytest.raises(q.QcfgError) as e:
                call(out=out, dtype=other)
            assert e.value.status == q.EINVAL
        assert not out.any()
        assert call(out=out, dtype=torch.float16) is out and torch.equal(out, call(dtype=torch.float16))
        call(out=out.zero_())
        assert torch.equal(out, call(dtype=torch.float16))
    assert ctx.linear_i8(x, w, s).dtype == torch.bfloat16 and ctx.gemm_i8_token(codes, w, 64, sx, s).dtype == torch.float32
    ctx.check_sync()


def test_the_largest_score_scale(ctx):
    """Scales are multiplied with log2(e) in fp32: one for which that is no number is refused, the largest one works."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(59)
    pool, cache, po, co = make(ctx, 8, 16, 2, 4, 2, 64)
    steps(ctx, pool, cache, po, co, [0], [20], torch.float32, rng, spread=0.1)
    x = torch.zeros((1, 2, 64), device="cuda")
    for scale in (2.0 ** 127, 2.5e38, float("inf"), float("nan"), 0.0, -1.0):
        with pytest.raises(q.QcfgError) as e:
            cache.attention(x, ints([0]), sm_scale=scale)
        assert e.value.status == q.EINVAL
    out = host(cache.attention(x, ints([0]), sm_scale=2.0 ** 126))
    want, tol = attention_bound(host(x), *co.values(0), 1.0, True, 0, torch.float32)      # all scores are 0
    assert (np.abs(out - want) <= tol).all()
    ctx.check_sync()


def test_a_batch_of_more_blocks_than_a_grid_has(ctx):
    """A million entries, mostly empty, of 4096 heads: the kernel for many rows would need more than 2^31 blocks."""
    rng = np.random.default_rng(61)
    n, heads, dim, rows = 1 << 20, 4096, 64, 256
    pool, cache, po, co = make(ctx, 2, 128, 2, 2, 1, dim)      # the oracle holds one head
    import paper_2302_01382_b200 as q
    cache = q.KvCache(pool, heads, dim)
    k, v = (rng.standard_normal((rows, 1, dim)).astype(np.float32) for _ in range(2))
    seqs, st = ints([1]), ints([0, rows])
    pool.extend(seqs, st)
    cache.append(dev(k).expand(-1, heads, -1).contiguous(), dev(v).expand(-1, heads, -1).contiguous(), seqs, st)
    assert po.extend([1], [rows])
    co.append(k, v, [1], [0, rows])
    x = rng.standard_normal((rows, 1, dim)).astype(np.float32)
    xd = dev(x, torch.float16)
    many = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    starts = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    many[-1], starts[-1] = 1, rows
    out = cache.attention(xd.expand(-1, heads, -1).contiguous(), many, starts, max_new=rows)
    ctx.check_sync()
    want, tol = attention_bound(host(xd), *co.values(1), dim ** -0.5, True, 0, torch.float16)
    assert (np.abs(host(out) - want) <= tol).all()             # every head (parts are cut at other places: not the same bits)


@pytest.mark.parametrize("m,k,n", [(65, 100, 18945), (68, 817, 21776), (77, 1, 25749), (100, 257, 32001), (128, 1000, 50257)])
@pytest.mark.parametrize("dtype,act,with_bias", [(torch.float32, "none", False), (torch.float16, "gelu", True)])
def test_linear_of_one_row_of_tiles_into_many_columns(ctx, m, k, n, dtype, act, with_bias):
    """65 to 128 tokens into more columns than tiles of 128 cover on 148 SMs."""
    linear_against_oracle(ctx, m, k, n, dtype, act, with_bias)


@pytest.mark.parametrize("m,k,n", [(100, 96, 20000), (300, 100, 700), (1000, 300, 4001), (1500, 64, 6000)])
def test_linear_without_pairs_of_ctas(m, k, n):
    import paper_2302_01382_b200 as q
    c = q.Context(0)
    try:
        c.set_pair_tiles(False)
        linear_against_oracle(c, m, k, n, torch.bfloat16, "relu", True)
    finally:
        c.close()


@pytest.mark.parametrize("m,k,n", [(1, 64, 51), (24, 2304, 9001), (33, 100, 1), (100, 257, 1557), (211, 141, 20003), (949, 22, 2310), (1756, 1085, 5)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_writes_no_column_behind_the_last(ctx, m, k, n, dtype):
    """Outputs on 16-byte boundaries, rows too, that end inside 16 bytes: what lies behind belongs to somebody else."""
    rng = np.random.default_rng(m + n)
    x = dev(rng.standard_normal((m, k)).astype(np.float32), dtype)
    w, sw = code_weights(rng, n, (k + 15) // 16 * 16)
    w[:, k:] = 0
    room = torch.full((m + 2, (n + 7) // 8 * 8 + 16), 7.0, dtype=dtype, device="cuda")
    bias = torch.ones(n, device="cuda")
    ctx.linear_i8(x, w, sw, bias=bias, out=room[1:m + 1, 8:8 + n])
    assert torch.equal(room[1:m + 1, 8:8 + n], ctx.linear_i8(x, w, sw, bias=bias))
    room[1:m + 1, 8:8 + n] = 7
    assert (room == 7).all()
    ctx.check_sync()
