"""The 8-bit serving operators against their oracle: linear layers quantized token by token, the paged cache, its attention.

Integers (codes, tables, counts) must be equal.  Tolerances of computed values count the roundings made: u = 2^-24 for an fp32
operation, half a step of the output's type (`torch.finfo(t).eps / 2`) for the final rounding.
"""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = {"none": 0, "relu": 1, "gelu": 2}


@pytest.fixture(scope="module")
def ctx():
    import paper_2302_01382_b200 as q
    c = q.Context(0)
    yield c
    c.close()


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ----------------------------------------------------------------------------- linear layers

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 768), (3, 17), (24, 4096), (65, 1001), (130, 16), (7, 20011)])
@pytest.mark.parametrize("bits", [8, 3])
def test_token_codes_bit_exact(ctx, dtype, shape, bits):
    rng = np.random.default_rng(shape[0] + shape[1])
    x = dev((rng.standard_normal(shape) * 10.0 ** rng.uniform(-3, 3, (shape[0], 1))).astype(np.float32), dtype)
    x[-1, :] = 0
    q, s = ctx.quantize_tokens(x, bits)
    qo, s_o = so.quantize_tokens(host(x), bits)
    np.testing.assert_array_equal(host(q)[:, :shape[1]], qo)
    assert not host(q)[:, shape[1]:].any()
    np.testing.assert_array_equal(host(s), s_o)
    if shape[1] > 8:                               # a strided view that begins off any 16-byte boundary
        v = x[:, 3:shape[1] - 2]
        q, s = ctx.quantize_tokens(v, bits, ldq=(shape[1] + 15) // 16 * 16 + 16)
        qo, s_o = so.quantize_tokens(host(v), bits)
        np.testing.assert_array_equal(host(q)[:, :v.shape[1]], qo)
        assert not host(q)[:, v.shape[1]:].any()
        np.testing.assert_array_equal(host(s), s_o)
    ctx.check_sync()


def test_token_codes_of_nonfinite_rows(ctx):
    import paper_2302_01382_b200 as q
    x = np.array([[1.0, np.nan, -2.0, np.inf], [0.5, 0.25, 0, -1], [1e-38, 0.0, -1e-38, 5e-39]], np.float32)
    codes, s = ctx.quantize_tokens(dev(x))
    assert ctx.sync_status() == q.ENONFINITE and ctx.sync_status() == q.OK
    qo, s_o = so.quantize_tokens(x)
    np.testing.assert_array_equal(host(codes)[:, :4], qo)
    np.testing.assert_array_equal(host(s), s_o)


def linear_bound(qx, sx, qw, sw, bias, act, dtype):
    """|error| of the kernel: float(acc), sx*sw, their product and the bias are one fp32 rounding each; relu passes an error on,
    tanh-GELU at most 1.13 times, adding its own 1e-6 of |y| with a floor of 1e-6 of the largest output."""
    lin = np.abs(so.linear(qx, sx, qw, sw))
    y = so.linear(qx, sx, qw, sw, bias, act)
    pre = 3.1 * U * lin + U * (lin + (0 if bias is None else np.abs(bias)))
    if act == "gelu":
        pre = 1.13 * pre + 1e-6 * np.abs(y) + 1e-6 * np.abs(y).max()
    return y, pre * (1 + half_step(dtype)) + half_step(dtype) * np.abs(y) + (2.0 ** -25 if dtype == torch.float16 else 1e-38)


LINEAR = [(1, 16, 16), (1, 768, 768), (2, 100, 33), (5, 4096, 1000), (8, 1024, 4096), (9, 777, 515), (16, 2048, 300), (17, 1024, 700), (24, 4096, 2048),
          (33, 515, 1030), (64, 1024, 1024), (65, 96, 70), (100, 2000, 40), (129, 1001, 259), (300, 768, 3072), (513, 3072, 768), (1037, 401, 2311)]


@pytest.mark.parametrize("m,k,n", LINEAR)
@pytest.mark.parametrize("dtype,act,with_bias", [(torch.float32, "none", False), (torch.bfloat16, "gelu", True), (torch.float16, "relu", True)])
def test_linear(ctx, m, k, n, dtype, act, with_bias):
    rng = np.random.default_rng(m * 31 + n)
    x = dev(rng.standard_normal((m, k)).astype(np.float32), dtype)
    w = rng.integers(-127, 128, (n, (k + 15) // 16 * 16)).astype(np.int8)
    w[:, k:] = 0
    sw = rng.uniform(0.5, 2, n).astype(np.float32) / np.float32(127 * np.sqrt(k))
    bias = rng.standard_normal(n).astype(np.float32) if with_bias else None
    bd = None if bias is None else dev(bias)
    y = ctx.linear_i8(x, dev(w), dev(sw), bias=bd, act=ACTS[act])
    qx, sx = so.quantize_tokens(host(x))
    want, tol = linear_bound(qx, sx, w[:, :k], sw, bias, act, dtype)
    assert (np.abs(host(y) - want) <= tol).all()
    # the two steps on their own give the same bits, into another type too
    codes, s = ctx.quantize_tokens(x)
    assert torch.equal(ctx.gemm_i8_token(codes, dev(w), k, s, dev(sw), bias=bd, act=ACTS[act], dtype=dtype), y)
    other = torch.float16 if dtype == torch.float32 else torch.float32
    want, tol = linear_bound(qx, sx, w[:, :k], sw, bias, act, other)
    assert (np.abs(host(ctx.linear_i8(x, dev(w), dev(sw), bias=bd, act=ACTS[act], dtype=other)) - want) <= tol).all()
    ctx.check_sync()


@pytest.mark.parametrize("m,k,n", [(1280, 300, 3136), (1280, 300, 2240), (1100, 130, 2311), (2000, 64, 2250), (257, 64, 16000)])
@pytest.mark.parametrize("dtype,act,with_bias", [(torch.float32, "relu", True), (torch.float16, "none", False)])
def test_linear_in_tiles_of_any_width(ctx, m, k, n, dtype, act, with_bias):
    """Sizes whose tiles are 224, 160, 192 and other numbers of columns wide on 148 SMs."""
    test_linear(ctx, m, k, n, dtype, act, with_bias)


@pytest.mark.parametrize("m", [1, 7, 40, 260])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_strided_rows_in_and_out(ctx, m, dtype):
    rng = np.random.default_rng(m)
    k, n = 333, 271
    wide = dev(rng.standard_normal((m, k + 10)).astype(np.float32), dtype)
    x = wide[:, 5:5 + k]
    w = np.zeros((n, 352), np.int8)
    w[:, :k] = rng.integers(-127, 128, (n, k))
    sw = np.full(n, 1e-3, np.float32)
    room = torch.full((m + 2, n + 9), 7.0, dtype=dtype, device="cuda")
    out = room[1:m + 1, 3:3 + n]
    ctx.linear_i8(x, dev(w), dev(sw), out=out)
    qx, sx = so.quantize_tokens(host(x))
    want, tol = linear_bound(qx, sx, w[:, :k], sw, None, "none", dtype)
    assert (np.abs(host(out) - want) <= tol).all()
    room[1:m + 1, 3:3 + n] = 7
    assert (room == 7).all()                       # nothing beside the output was written
    ctx.check_sync()


def test_linear_narrow_grids_and_empty_batches(ctx):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 64)).astype(np.float32)
    w = rng.integers(-7, 8, (48, 64)).astype(np.int8)
    sw = np.full(48, 0.01, np.float32)
    for bits in range(2, 9):
        y = ctx.linear_i8(dev(x), dev(w), dev(sw), bits=bits)
        qx, sx = so.quantize_tokens(x, bits)
        want, tol = linear_bound(qx, sx, w, sw, None, "none", torch.float32)
        assert (np.abs(host(y) - want) <= tol).all()
    assert ctx.linear_i8(dev(x)[:0], dev(w), dev(sw)).shape == (0, 48)
    # the largest sums int32 holds: 131072 products of 127 * 127
    x = torch.ones((2, 131072), device="cuda")
    w = torch.full((3, 131072), 127, dtype=torch.int8, device="cuda")
    y = ctx.linear_i8(x, w, torch.ones(3, device="cuda"))
    assert (np.abs(host(y) / (131072 * 127.0) - 1) <= 4 * U).all()


def test_linear_refusals(ctx):
    import paper_2302_01382_b200 as q
    x = torch.ones((4, 64), device="cuda")
    w = torch.ones((32, 64), dtype=torch.int8, device="cuda")
    s = torch.ones(32, device="cuda")
    for bad, status in [(lambda: ctx.linear_i8(x, w, s, bits=9), q.EBITS), (lambda: ctx.linear_i8(x, w, s, bits=1), q.EBITS),
                        (lambda: ctx.linear_i8(x, w, s, act=3), q.EINVAL), (lambda: ctx.linear_i8(x.double(), w, s), q.EINVAL),
                        (lambda: ctx.linear_i8(x, w[:, :48], s), q.ESHAPE), (lambda: ctx.linear_i8(x, w, s[:31]), q.ESHAPE),
                        (lambda: ctx.linear_i8(x, w, s, out=x), q.ESHAPE), (lambda: ctx.linear_i8(x.T, w, s), q.ESHAPE),
                        (lambda: ctx.linear_i8(x[:, :40], torch.ones((32, 72), dtype=torch.int8, device="cuda")[:, 1:41], s), q.EALIGN),
                        (lambda: ctx.quantize_tokens(x, ldq=72), q.EALIGN), (lambda: ctx.quantize_tokens(x, ldq=48), q.ESHAPE),
                        (lambda: ctx.linear_i8(x.cpu(), w, s), q.EINVAL)]:
        with pytest.raises(q.QcfgError) as e:
            bad()
        assert e.value.status == status
    long = torch.ones((1, 131088), device="cuda")
    with pytest.raises(q.QcfgError):
        ctx.linear_i8(long, torch.ones((1, 131088), dtype=torch.int8, device="cuda"), s[:1])


# ----------------------------------------------------------------------------- pages

def make(ctx, n_pages, page, max_seqs, max_pages, heads=2, dim=64):
    import paper_2302_01382_b200 as q
    pool = q.KvPool(ctx, n_pages, page, max_seqs, max_pages)
    po = so.Pool(n_pages, page, max_seqs, max_pages)
    return pool, q.KvCache(pool, heads, dim), po, so.Cache(po, heads, dim)


def starts_of(rows):
    return [0] + list(np.cumsum(rows))


def same_pool(pool, po):
    np.testing.assert_array_equal(host(pool.table), po.table_array())
    np.testing.assert_array_equal(host(pool.lens), po.lens)
    np.testing.assert_array_equal(host(pool.refs), po.refs)


def same_cache(cache, co):
    """Every page in use holds the same codes in its filled rows and the same maxima."""
    po = co.pool
    for z, (c, a) in enumerate(((cache.k, cache.k_absmax), (cache.v, cache.v_absmax))):
        c, a = host(c), host(a)
        for s in range(po.max_seqs):
            for j, p in enumerate(po.table[s]):
                rows = min(po.page, po.lens[s] - j * po.page)
                np.testing.assert_array_equal(a[p], co.absmax[z][p])
                np.testing.assert_array_equal(c[p, :, :rows], co.codes[z][p, :, :rows])


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_pages_through_a_long_run(ctx, page):
    """Sequences come, grow, fork, leave and are compacted in random order; after every call all numbers are the oracle's."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(page)
    n_pages, max_seqs, max_pages = 210, 23, 14
    pool, cache, po, co = make(ctx, n_pages, page, max_seqs, max_pages)
    # give every page contents of its own, so that a wrong copy shows
    for z, (c, a) in enumerate(((cache.k, cache.k_absmax), (cache.v, cache.v_absmax))):
        co.codes[z][:] = rng.integers(-127, 128, co.codes[z].shape)
        co.absmax[z][:] = rng.uniform(0.1, 4, co.absmax[z].shape)
        c.copy_(dev(co.codes[z]))
        a.copy_(dev(co.absmax[z]))
    refused = 0
    for _ in range(120):
        what = rng.integers(0, 10)
        if what < 5:
            seqs = rng.permutation(max_seqs)[:rng.integers(1, 8)]
            seqs = np.where(rng.random(len(seqs)) < 0.1, -1, seqs)
            rows = rng.integers(0, 4 * page, len(seqs)) if rng.random() < 0.7 else np.ones(len(seqs), int)
            pool.extend(ints(seqs), ints(starts_of(rows)))
            ok = po.extend(list(seqs), list(rows))
            refused += not ok
            assert ctx.sync_status() == (q.OK if ok else q.EPAGE)
        elif what < 7:
            seqs = rng.integers(-1, max_seqs, rng.integers(1, 6))
            pool.free(ints(seqs))
            po.free(list(seqs))
        elif what < 9:
            n = rng.integers(1, 6)
            parents, children = rng.integers(0, max_seqs, n), rng.permutation(max_seqs)[:n]
            if rng.random() < 0.6:
                empty = [s for s in range(max_seqs) if po.lens[s] == 0][:n]
                children = np.array(empty + [-1] * (n - len(empty)))
            src, dst = pool.fork(ints(parents), ints(children))
            want = po.fork(list(parents), list(children))
            assert ctx.sync_status() == (q.OK if want else q.EPAGE)
            refused += want is None
            cache.copy_pages(src, dst)
            if want:
                assert host(src).tolist() == want[0] and host(dst).tolist() == want[1]
                co.copy_pages(*want)
            else:
                assert (host(src) == -1).all() and (host(dst) == -1).all()
        else:
            where = pool.compact()
            want = po.compact()
            assert host(where).tolist() == want
            cache.copy_pages(None, where)
            co.copy_pages(None, want)
        same_pool(pool, po)
    same_cache(cache, co)
    assert refused > 3
    ctx.check_sync()


def test_large_pools(ctx):
    """More pages than one walk of a block covers, more entries than it has threads, and tables of many rows."""
    import paper_2302_01382_b200 as q
    n_pages, max_seqs = 20000, 3000
    pool, po = q.KvPool(ctx, n_pages, 16, max_seqs, 9), so.Pool(n_pages, 16, max_seqs, 9)
    rng = np.random.default_rng(3)
    rows = rng.integers(0, 140, max_seqs)
    pool.extend(ints(range(max_seqs)), ints(starts_of(rows)))
    assert po.extend(list(range(max_seqs)), list(rows))
    same_pool(pool, po)
    gone = rng.permutation(max_seqs)[:1500]
    pool.free(ints(gone))
    po.free(list(gone))
    parents = np.setdiff1d(np.arange(max_seqs), gone)
    src, dst = pool.fork(ints(parents), ints(gone))
    want = po.fork(list(parents), list(gone))
    assert host(src).tolist() == want[0] and host(dst).tolist() == want[1]
    pool.free(ints(parents[::2]))
    po.free(list(parents[::2]))
    assert host(pool.compact()).tolist() == po.compact()
    same_pool(pool, po)
    ctx.check_sync()


def test_pages_with_numbers_out_of_range(ctx):
    import paper_2302_01382_b200 as q
    pool, cache, po, _ = make(ctx, 8, 16, 3, 4)
    pool.extend(ints([0]), ints([0, 20]))
    po.extend([0], [20])
    ctx.check_sync()
    for bad in (lambda: pool.extend(ints([1, 3]), ints([0, 1, 2])), lambda: pool.extend(ints([1, 1])), lambda: pool.extend(ints([1]), ints([0, 65])),
                lambda: pool.free(ints([3])), lambda: pool.fork(ints([5]), ints([1])), lambda: pool.fork(ints([0]), ints([3])),
                lambda: pool.fork(ints([0, 0]), ints([1, 1])), lambda: pool.fork(ints([1]), ints([0])),
                lambda: cache.copy_pages(ints([8]), ints([1])), lambda: cache.copy_pages(ints([1]), ints([9]))):
        bad()
        assert ctx.sync_status() == q.EPAGE
        same_pool(pool, po)
    cache.copy_pages(ints([-1, 2, 3]), ints([1, -1, 3]))
    ctx.check_sync()


# ----------------------------------------------------------------------------- writing and reading

def steps(ctx, pool, cache, po, co, seqs, rows, dtype, rng, spread=1.0, behind=0, layout="rows"):
    """One extend + append on both sides."""
    n = sum(rows) + behind
    shape = (n, cache.kv_heads, cache.head_dim)
    k, v = ((rng.standard_normal(shape) * spread).astype(np.float32) for _ in range(2))
    kd, vd = dev(k, dtype), dev(v, dtype)
    if layout == "packed":                         # columns of one projection
        both = torch.cat([kd.flatten(1), vd.flatten(1)], 1)
        kd, vd = (t.unflatten(1, shape[1:]) for t in both.split(shape[1] * shape[2], 1))
    elif layout == "heads":                        # [heads, rows, dim]
        kd, vd = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (kd, vd))
    st = ints(starts_of(rows))
    pool.extend(ints(seqs), st)
    cache.append(kd, vd, ints(seqs), st)
    assert po.extend(list(seqs), list(rows))
    co.append(host(kd), host(vd), list(seqs), starts_of(rows))


@pytest.mark.parametrize("page,heads,dim", [(16, 1, 16), (32, 3, 80), (64, 2, 64), (64, 8, 128), (128, 2, 256)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_append_and_read(ctx, page, heads, dim, dtype):
    """Prompts, then tokens one by one whose size grows, so that pages change their grid; rows behind the last are not read."""
    rng = np.random.default_rng(page + dim)
    pool, cache, po, co = make(ctx, 60, page, 6, 12, heads, dim)
    steps(ctx, pool, cache, po, co, [0, 1, -1, 2], [page + 3, 0, 5, 2 * page], dtype, rng, behind=3)
    for t in range(6):
        steps(ctx, pool, cache, po, co, [2, 0, 3], [1, 1, t], dtype, rng, spread=1 + t, layout=["rows", "packed", "heads"][t % 3])
    same_pool(pool, po)
    same_cache(cache, co)
    # every token, some behind the end, an entry without a sequence, rows behind the last entry
    for out_type in DTYPES:
        counts = [po.lens[0] + 2, 4, po.lens[3], po.lens[2] - 5]
        seqs, first = [0, -1, 3, 2], [0, 0, 0, 5]
        k, v = cache.read(ints(seqs), ints(first), ints(starts_of(counts)), sum(counts), out_type)
        for z, got in enumerate((host(k), host(v))):
            at = 0
            for s, f, c in zip(seqs, first, counts):
                want = co.values(s)[z][f:f + c] if s >= 0 else np.zeros((0, heads, dim))
                mine = got[at:at + c]
                assert (np.abs(mine[:len(want)] - want) <= (U + half_step(out_type)) * np.abs(want) + 2.0 ** -25).all()
                assert not mine[len(want):].any()
                at += c
    ctx.check_sync()


def test_append_nonfinite_values_stay_with_their_token(ctx):
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(0)
    pool, cache, po, co = make(ctx, 4, 16, 1, 4)
    x = rng.standard_normal((20, 2, 64)).astype(np.float32)
    x[3, 0, 5], x[4, 1, 6], x[18, 0, :] = np.nan, -np.inf, np.inf
    pool.extend(ints([0]), ints([0, 20]))
    cache.append(dev(x), dev(-x), ints([0]), ints([0, 20]))
    assert ctx.sync_status() == q.ENONFINITE
    po.extend([0], [20])
    co.append(x, -x, [0], [0, 20])
    same_cache(cache, co)
    ctx.check_sync()


def test_append_writes_no_page_it_must_not(ctx):
    """Shared pages, sequences listed twice and table entries out of range are left out and reported; the others are written."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(1)
    pool, cache, po, co = make(ctx, 12, 16, 5, 4)
    steps(ctx, pool, cache, po, co, [0, 1, 2], [20, 20, 20], torch.float32, rng)
    ctx.check_sync()
    before = [t.clone() for t in (cache.k, cache.v, cache.k_absmax, cache.v_absmax)]
    x = dev(rng.standard_normal((3, 2, 64)).astype(np.float32))
    pool.refs[po.table[0][1]] = 2                  # held by another sequence too
    pool.table[1, 1] = 12                          # no such page
    pool.extend(ints([0, 1]))
    cache.append(x[:2], x[:2], ints([0, 1]))
    assert ctx.sync_status() == q.EPAGE
    pool.table[1, 1] = -1
    cache.append(x[:1], x[:1], ints([1]))
    assert ctx.sync_status() == q.EPAGE
    pool.extend(ints([2]))
    ctx.check_sync()
    cache.append(x, x, ints([2, 4, 2]))
    assert ctx.sync_status() == q.EPAGE
    cache.append(x[:1], x[:1], ints([5]))
    assert ctx.sync_status() == q.EPAGE
    for a, b in zip(before, (cache.k, cache.v, cache.k_absmax, cache.v_absmax)):
        assert torch.equal(a, b)
    cache.append(x[:1], x[:1], ints([2]))
    ctx.check_sync()
    assert not torch.equal(before[0], cache.k)


# ----------------------------------------------------------------------------- attention

def attention_bound(q, k, v, sm_scale, causal, window, dtype):
    """Oracle and |error|: a score is a sum of dim products and three scalings in fp32, with fp32 queries held to 2^-22 of their
    size and others to 2^-22 of their row's largest; an exponential and its argument cost 2^-21; the weights of the values are rounded to
    11 bits for 16-bit types (to 22 for fp32); sums over the tokens are fp32."""
    out, weight, spread = so.attention(q, k, v, sm_scale, causal, window)
    dim, length = q.shape[2], k.shape[0]
    biggest = np.abs(q).max(2, initial=0) * np.abs(k).sum(2).max(initial=0) * sm_scale
    score = (dim + 6) * U * spread + 2.0 ** -22 * (spread + biggest) + 2.0 ** -21
    p = 2.0 ** -11 if dtype != torch.float32 else 2.0 ** -20
    rel = 2 * np.expm1(score) + p + (length + 8) * U
    tiny = 2.0 ** -23 * np.abs(v).max(initial=0)   # weights below the fp16 grid
    return out, rel[:, :, None] * weight + half_step(dtype) * np.abs(out) + tiny + 2.0 ** -25


def check_attention(ctx, cache, co, seqs, rows, q_heads, dtype, rng, behind=0, layout="rows", **kw):
    n = sum(rows) + behind
    dim = cache.head_dim
    q = dev((rng.standard_normal((n, q_heads, dim)) * rng.uniform(0.3, 3, (n, 1, 1))).astype(np.float32), dtype)
    out = None
    if layout == "packed":
        q = torch.cat([q, q.new_zeros((n, 3, dim))], 1)[:, :q_heads]
        out = torch.full((n, q_heads + 1, dim), 9.0, dtype=dtype, device="cuda")[:, :q_heads]
    elif layout == "heads":
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
    if out is None:
        out = torch.full((n, q_heads, dim), 9.0, dtype=dtype, device="cuda")
    hints = {k: kw.pop(k) for k in ("max_new", "max_len") if k in kw}
    cache.attention(q, ints(seqs), ints(starts_of(rows)) if rows is not None else None, out=out, **kw, **hints)
    ctx.check_sync()
    got, at = host(out), 0
    scale = kw.get("sm_scale") or dim ** -0.5
    for s, c in zip(seqs, rows):
        if s >= 0:
            k, v = co.values(s)
            want, tol = attention_bound(host(q)[at:at + c], k, v, scale, kw.get("causal", True), kw.get("window", 0), dtype)
            worst = np.abs(got[at:at + c] - want) - tol
            assert (worst <= 0).all(), (s, c, float(worst.max()), np.argwhere(worst > 0)[:4].tolist())
        else:
            assert not got[at:at + c].any()
        at += c
    assert (got[at:] == 9).all()
    if layout == "packed":
        assert (out._base[:, q_heads:] == 9).all()
    return q, out


CACHES = [(16, 12, 12, 64), (64, 8, 2, 64), (32, 7, 1, 128), (128, 4, 4, 128), (64, 32, 2, 128), (16, 3, 3, 80), (32, 4, 2, 256), (64, 40, 1, 16), (16, 24, 2, 96)]


@pytest.mark.parametrize("page,q_heads,heads,dim", CACHES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_of_single_tokens(ctx, page, q_heads, heads, dim, dtype):
    rng = np.random.default_rng(page * dim + q_heads)
    lens = [1, page - 1, page, page + 1, 0, 3 * page + 5, 700, 257]
    pool, cache, po, co = make(ctx, 200, page, 9, 800 // page + 1, heads, dim)
    steps(ctx, pool, cache, po, co, list(range(8)), lens, dtype, rng, spread=2.0)
    order = [6, 0, -1, 4, 5, 2, 1, 7, 3, 6]        # any order, a padded entry, an empty sequence, one listed twice
    ones = [1] * len(order)
    check_attention(ctx, cache, co, order, ones, q_heads, dtype, rng)
    check_attention(ctx, cache, co, order, ones, q_heads, dtype, rng, behind=3, layout="packed", max_new=1, max_len=700)
    check_attention(ctx, cache, co, order, ones, q_heads, dtype, rng, layout="heads", window=page + 2, sm_scale=0.3)
    check_attention(ctx, cache, co, [6], [1], q_heads, dtype, rng, causal=False)
    check_attention(ctx, cache, co, order, ones, q_heads, dtype, rng, max_new=1, max_len=300)      # a hint that is wrong


@pytest.mark.parametrize("page,q_heads,heads,dim", CACHES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_of_prompts(ctx, page, q_heads, heads, dim, dtype):
    """Ragged queries behind contexts of any length: more queries than tokens (rows that see nothing), one query, none, many."""
    rng = np.random.default_rng(page * dim + heads)
    lens = [300, 5, page, 131, 0, 64]
    pool, cache, po, co = make(ctx, 120, page, 6, 320 // page + 1, heads, dim)
    steps(ctx, pool, cache, po, co, list(range(6)), lens, dtype, rng, spread=2.0)
    seqs, rows = [3, 0, -1, 1, 4, 2, 5], [130, 37, 6, 9, 4, 0, 1]
    check_attention(ctx, cache, co, seqs, rows, q_heads, dtype, rng)
    check_attention(ctx, cache, co, seqs, rows, q_heads, dtype, rng, behind=5, layout="packed", max_new=130, max_len=300)
    check_attention(ctx, cache, co, seqs, rows, q_heads, dtype, rng, layout="heads", window=33)
    check_attention(ctx, cache, co, seqs, rows, q_heads, dtype, rng, causal=False, max_new=130)
    check_attention(ctx, cache, co, [0], [300], q_heads, dtype, rng, window=1)


MANY = [(16, 12, 12, 64, [torch.float32, torch.bfloat16, torch.float16]), (128, 16, 8, 64, DTYPES), (64, 32, 8, 128, DTYPES[1:]), (32, 56, 8, 128, DTYPES[1:]),
        (16, 8, 8, 128, DTYPES[1:]), (64, 130, 5, 128, DTYPES[1:])]


@pytest.mark.parametrize("page,q_heads,heads,dim,dtypes", MANY)
def test_attention_of_many_rows(ctx, page, q_heads, heads, dim, dtypes):
    """Enough rows for the kernel that takes 256 at a time: ragged entries, rows that see nothing, windows, contexts that end anywhere."""
    group = q_heads // heads
    lens = [530, 129, 5, 700, 0, 257, 1, 384, 40, 256]
    rows = [400, 129, 9, 128, 3, 257, 1, 300, 0, 255]
    for dtype in dtypes:
        rng = np.random.default_rng(page + group)
        pool, cache, po, co = make(ctx, 2600 // page + 30, page, len(lens), 704 // page + 1, heads, dim)
        steps(ctx, pool, cache, po, co, list(range(len(lens))), lens, dtype, rng, spread=2.0)
        order = [3, 0, -1, 1, 2, 4, 5, 6, 7, 8, 9]
        counts = [rows[s] if s >= 0 else 2 for s in order]
        for kw in ({}, {"behind": 5, "layout": "packed", "max_new": 400}, {"layout": "heads", "window": 100}, {"causal": False}, {"window": 3, "sm_scale": 1.0}):
            before = ctx.launch_count()
            check_attention(ctx, cache, co, order, counts, q_heads, dtype, rng, **kw)
            # max_new unknown: the mean decides, 135 rows here
            assert ctx.launch_count() - before == (1 if "max_new" in kw or 135 * group >= (64 if dim == 64 else 32) else 2)


def test_many_entries_and_heads(ctx):
    """More entries than a block has threads, in every kernel that looks for its own; more heads than a warp has lanes."""
    rng = np.random.default_rng(41)
    n, heads = 500, 40
    lens = [int(v) for v in rng.integers(0, 21, n)]
    pool, cache, po, co = make(ctx, 2 * n, 16, n, 3, heads, 16)
    order = [int(v) for v in rng.permutation(n)]
    steps(ctx, pool, cache, po, co, order, [lens[s] for s in order], torch.bfloat16, rng)
    steps(ctx, pool, cache, po, co, order[::-1], [1] * n, torch.bfloat16, rng, spread=2.0)
    same_pool(pool, po)
    same_cache(cache, co)
    counts = [po.lens[s] for s in order]
    k, v = cache.read(ints(order), ints([0] * n), ints(starts_of(counts)), sum(counts))
    for z, got in enumerate((host(k), host(v))):
        want = np.concatenate([co.values(s)[z] for s in order])
        assert (np.abs(got - want) <= (U + half_step(torch.float32)) * np.abs(want) + 2.0 ** -25).all()
    check_attention(ctx, cache, co, order, [min(2, po.lens[s]) for s in order], heads, torch.bfloat16, rng)
    check_attention(ctx, cache, co, order, [min(2, po.lens[s]) for s in order], 2 * heads, torch.bfloat16, rng, max_len=22)
    # the kernel for many rows: the hint says so
    n = 420
    lens = [int(v) for v in rng.integers(0, 6, n)]
    lens[399] = 230
    pool, cache, po, co = make(ctx, n + 20, 64, n, 4, 1, 64)
    steps(ctx, pool, cache, po, co, list(range(n)), lens, torch.float16, rng)
    before = ctx.launch_count()
    check_attention(ctx, cache, co, list(range(n)), [min(v, 200) for v in lens], 2, torch.float16, rng, max_new=200)
    assert ctx.launch_count() - before == 1


def test_attention_of_uneven_scales(ctx):
    """Pages whose maxima differ by ten orders of magnitude, values of zero pages, scores up to hundreds."""
    for dtype in DTYPES:
        rng = np.random.default_rng(7)
        pool, cache, po, co = make(ctx, 40, 16, 2, 40, 25, 64)
        for t in range(12):
            steps(ctx, pool, cache, po, co, [0], [16], torch.float32, rng, spread=0.0 if t % 5 == 4 else 10.0 ** (t - 8))
        check_attention(ctx, cache, co, [0], [1], 50, dtype, rng, sm_scale=0.02)
        check_attention(ctx, cache, co, [0], [20], 50, dtype, rng, sm_scale=0.02)
        check_attention(ctx, cache, co, [0, 0], [150, 100], 50, dtype, rng, sm_scale=0.02, max_new=150)


def test_attention_of_a_long_context(ctx):
    rng = np.random.default_rng(11)
    pool, cache, po, co = make(ctx, 700, 64, 3, 400, 2, 128)
    steps(ctx, pool, cache, po, co, [0, 1], [20011, 9], torch.bfloat16, rng)
    check_attention(ctx, cache, co, [1, 0], [1, 1], 8, torch.bfloat16, rng)
    check_attention(ctx, cache, co, [0], [3], 8, torch.float16, rng, max_new=3)
    check_attention(ctx, cache, co, [0], [1], 8, torch.float32, rng, window=9000)


def test_attention_offsets_beyond_32_bits(ctx):
    """Pages whose byte offsets do not fit 32 bits (a 4.9 GB cache) are written, read and attended to."""
    import paper_2302_01382_b200 as q
    heads, dim, page, n_pages = 8, 128, 128, 18700
    pool = q.KvPool(ctx, n_pages, page, 2, 3)
    k = torch.zeros((n_pages, heads, page, dim), dtype=torch.int8, device="cuda")
    cache = q.KvCache(pool, heads, dim, k=k, v=k.clone())
    po = so.Pool(4, page, 1, 3)
    co = so.Cache(po, heads, dim)
    rng = np.random.default_rng(2)
    far = [n_pages - 1, 17000, n_pages - 2]
    pool.table[1] = ints(far)
    pool.refs[ints(far).long()] = 1
    pool.lens[1] = 300
    x = [dev(rng.standard_normal((300, heads, dim)).astype(np.float32)) for _ in range(2)]
    cache.append(*x, ints([1]), ints([0, 300]))
    po.extend([0], [300])
    co.append(host(x[0]), host(x[1]), [0], [0, 300])
    for j, p in enumerate(far):
        rows = min(page, 300 - j * page)
        np.testing.assert_array_equal(host(cache.k[p])[:, :rows], co.codes[0][po.table[0][j]][:, :rows])
    for dtype, rows in ((torch.bfloat16, 1), (torch.bfloat16, 200), (torch.float32, 5)):
        qs = dev(rng.standard_normal((rows, 16, dim)).astype(np.float32), dtype)
        out = cache.attention(qs, ints([1]), ints([0, rows]))
        want, tol = attention_bound(host(qs), *co.values(0), dim ** -0.5, True, 0, dtype)
        assert (np.abs(host(out) - want) <= tol).all()
    cache.copy_pages(ints([n_pages - 1]), ints([18000]))
    assert torch.equal(cache.v[18000], cache.v[n_pages - 1])
    ctx.check_sync()


def test_attention_of_nonfinite_queries_and_bad_pages(ctx):
    """A query with NaN spoils its own rows only; tokens on pages that do not exist are left out and reported."""
    import paper_2302_01382_b200 as q
    for dtype in DTYPES:
        for rows, heads in ((1, 2), (40, 2), (100, 26)):
            rng = np.random.default_rng(13)
            pool, cache, po, co = make(ctx, 30, 16, 3, 8, heads, 64)
            steps(ctx, pool, cache, po, co, [0, 1], [100, 50], torch.float32, rng)
            x = dev(rng.standard_normal((2 * rows, 2 * heads, 64)).astype(np.float32), dtype)
            clean = cache.attention(x, ints([0, 1]), ints([0, rows, 2 * rows]))
            y = x.clone()
            y[0, 1, 3] = float("nan")
            got = cache.attention(y, ints([0, 1]), ints([0, rows, 2 * rows]))
            assert got[0, 1].isnan().all()
            got[0, 1] = clean[0, 1]
            assert torch.equal(got, clean)
            ctx.check_sync()
            pool.table[0, 2] = 30
            pool.table[0, 3] = -5
            got = cache.attention(x, ints([0, 1]), ints([0, rows, 2 * rows]))
            assert ctx.sync_status() == q.EPAGE
            assert torch.equal(got[rows:], clean[rows:]) and got[:rows].isfinite().all()
            got = cache.attention(x, ints([7, 1]), ints([0, rows, 2 * rows]))
            assert ctx.sync_status() == q.EPAGE
            assert torch.equal(got[rows:], clean[rows:]) and not got[:rows].any()


@pytest.mark.parametrize("dim,dtype", [(64, torch.float32), (64, torch.bfloat16), (128, torch.float16)])
def test_many_rows_with_nonfinite_queries_and_bad_pages(ctx, dim, dtype):
    """In the kernel for many rows a NaN or Inf stays with its row, and a page that is not there with its sequence."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(dim)
    pool, cache, po, co = make(ctx, 80, 16, 3, 24, 16, dim)
    lens = [300, 257, 384]
    steps(ctx, pool, cache, po, co, [0, 1, 2], lens, dtype, rng)
    x = dev(rng.standard_normal((sum(lens), 16, dim)).astype(np.float32), dtype)
    seqs, starts = ints([0, 1, 2]), ints(starts_of(lens))
    run = lambda x: cache.attention(x, seqs, starts, max_new=384)
    before = ctx.launch_count()
    clean = run(x)
    assert ctx.launch_count() - before == 1
    bad = x.clone()
    bad[5, 3, 0], bad[299, 3, 7], bad[301, 11, dim - 1] = float("nan"), float("inf"), -float("inf")
    got = run(bad)
    ctx.check_sync()
    hit = torch.zeros(got.shape[:2], dtype=torch.bool, device="cuda")
    hit[5, 3] = hit[299, 3] = hit[301, 11] = True
    assert torch.isnan(got[hit].float()).all() and torch.equal(got[~hit], clean[~hit])
    streamed = cache.attention(bad, seqs, starts, max_new=1)
    assert torch.isnan(streamed[hit].float()).all() and torch.isfinite(streamed[~hit].float()).all()
    pool.table[1, 3] = 1 << 20
    pool.table[2, 0] = -1
    got = run(x)
    with pytest.raises(q.QcfgError) as e:
        ctx.check_sync()
    assert e.value.status == q.EPAGE
    assert torch.equal(got[:300], clean[:300]) and torch.isfinite(got.float()).all()
    # the rows in front of the page; the sequence's largest value scale may be that page's, so to the bits of the bound only
    k, v = (t[:48] for t in co.values(1))
    want, tol = attention_bound(host(x)[300:348], k, v, dim ** -0.5, True, 0, dtype)
    assert (np.abs(host(got)[300:348] - want) <= tol).all()
    assert not got[557:557 + 16].any()                               # these rows see that page only


def test_garbage_behind_the_end_is_not_seen(ctx):
    """Codes behind the last token and the maxima of pages nobody holds do not matter, whatever they are."""
    for dtype in DTYPES:
        rng = np.random.default_rng(17)
        pool, cache, po, co = make(ctx, 30, 64, 3, 8, 26, 64)
        cache.k.fill_(-128)
        cache.v.fill_(-128)
        cache.k_absmax.fill_(float("nan"))
        cache.v_absmax.fill_(float("inf"))
        steps(ctx, pool, cache, po, co, [0, 1], [70, 3], torch.float32, rng)
        check_attention(ctx, cache, co, [0, 1], [1, 1], 104, dtype, rng)
        check_attention(ctx, cache, co, [0, 1], [70, 3], 104, dtype, rng, max_new=70)
        check_attention(ctx, cache, co, [0, 1], [10, 2], 104, dtype, rng, causal=False)
        check_attention(ctx, cache, co, [0, 1], [65, 2], 104, dtype, rng, causal=False, max_new=65)


def test_repeats_give_the_same_bits(ctx):
    rng = np.random.default_rng(19)
    pool, cache, po, co = make(ctx, 400, 16, 8, 320, 2, 128)
    steps(ctx, pool, cache, po, co, list(range(4)), [4000, 17, 900, 1], torch.bfloat16, rng)
    for rows in ([1, 1, 1, 1], [5, 3, 7, 1], [3000, 17, 900, 1]):
        q = dev(rng.standard_normal((sum(rows), 16, 128)).astype(np.float32), torch.bfloat16)
        first = cache.attention(q, ints(range(4)), ints(starts_of(rows)))
        for _ in range(5):
            assert torch.equal(cache.attention(q, ints(range(4)), ints(starts_of(rows))), first)
    ctx.check_sync()


def test_attention_refusals(ctx):
    import paper_2302_01382_b200 as q
    pool, cache, _, _ = make(ctx, 8, 16, 3, 4, 2, 64)
    x = torch.ones((3, 4, 64), device="cuda")
    s, st = ints([0, 1]), ints([0, 1, 3])
    for bad, status in [(lambda: cache.attention(x, s, st, sm_scale=0.0), q.EINVAL), (lambda: cache.attention(x, s, st, sm_scale=float("nan")), q.EINVAL),
                        (lambda: cache.attention(x, s, st, window=-1), q.EINVAL), (lambda: cache.attention(x, s, st, causal=False, window=4), q.EINVAL),
                        (lambda: cache.attention(x[:, :3], s, st), q.ESHAPE), (lambda: cache.attention(x[:, :, :32], s, st), q.ESHAPE),
                        (lambda: cache.attention(x.double(), s, st), q.EINVAL), (lambda: cache.attention(x, s, st[:2]), q.EINVAL),
                        (lambda: cache.attention(x, s.long(), st), q.EINVAL), (lambda: cache.attention(x, s, st, out=x[:2]), q.ESHAPE),
                        (lambda: cache.attention(x.flatten()[1:1 + 2 * 256].view(2, 4, 64), s), q.EALIGN),
                        (lambda: cache.append(x[:, :2], x[:, :1], s, st), q.ESHAPE), (lambda: cache.append(x, x, s, st), q.ESHAPE),
                        (lambda: cache.append(x[:1, :2], x[:1, :2], s), q.ESHAPE), (lambda: cache.attention(x.cpu(), s, st), q.EINVAL),
                        (lambda: q.KvCache(pool, 2, 24).attention(x, s, st), q.ESHAPE), (lambda: q.KvPool(ctx, 8, 48, 3, 4).extend(s), q.ESHAPE),
                        (lambda: q.KvCache(pool, 2, 64, k=cache.k[:4]), q.ESHAPE), (lambda: cache.copy_pages(ints([1]), ints([1, 2])), q.EINVAL)]:
        with pytest.raises(q.QcfgError) as e:
            bad()
        assert e.value.status == status
    assert cache.attention(x[:0], s, ints([0, 0, 0])).shape == (0, 4, 64)
    assert cache.attention(x[:0], s[:0]).shape == (0, 4, 64)


def test_refusals_of_pools_beyond_32_bits_and_of_outputs_in_place(ctx):
    import paper_2302_01382_b200 as q
    pool, cache, _, _ = make(ctx, 8, 16, 3, 4, 2, 64)
    x = torch.ones((2, 4, 64), device="cuda")
    with pytest.raises(q.QcfgError) as e:
        cache.attention(x, ints([0, 1]), out=x)
    assert e.value.status == q.EINVAL
    for field, value in (("n_pages", 0x7fffffff), ("max_seqs", 0x7fffffff), ("max_pages", 0x7fffffff // 16)):
        before = getattr(pool._c, field)
        setattr(pool._c, field, value)
        for call in (lambda: pool.extend(ints([0])), lambda: pool.free(ints([0])), lambda: cache.attention(x, ints([0, 1]))):
            with pytest.raises(q.QcfgError) as e:
                call()
            assert e.value.status == q.ESHAPE
        setattr(pool._c, field, before)
    assert not cache.attention(x, ints([0, 1])).any()
    ctx.check_sync()


# ----------------------------------------------------------------------------- together

def block(ctx, cache, weights, x, seqs, starts, heads, group, dim):
    """Attention half of a transformer block as a decoder runs it."""
    qkv = ctx.linear_i8(x, *weights[0])
    q, k, v = qkv.split([heads * group * dim, heads * dim, heads * dim], 1)
    cache.append(k.unflatten(1, (heads, dim)), v.unflatten(1, (heads, dim)), seqs, starts)
    y = cache.attention(q.unflatten(1, (heads * group, dim)), seqs, starts)
    return ctx.linear_i8(y.flatten(1), *weights[1])


def code_weights(rng, n, k):
    return dev(rng.integers(-127, 128, (n, k)).astype(np.int8)), dev(rng.uniform(0.5, 1.5, n).astype(np.float32) / np.float32(73 * np.sqrt(k)))


@pytest.mark.parametrize("dtype", DTYPES)
def test_generation_prompt_fork_and_steps(ctx, dtype):
    """Prompts, forks, single steps, sequences that leave and a compaction: at every step the block's output is that of the oracle
    working on the same inputs, and a captured step replays with other lengths."""
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(23)
    heads, group, dim, hidden = 2, 4, 64, 256
    pool, cache, po, co = make(ctx, 90, 16, 8, 12, heads, dim)
    weights = [code_weights(rng, (group + 2) * heads * dim, hidden), code_weights(rng, hidden, group * heads * dim)]
    np_weights = [[host(t) for t in w] for w in weights]

    def step(seqs, rows, run=None):
        x = dev(rng.standard_normal((sum(rows), hidden)).astype(np.float32), dtype)
        st = starts_of(rows)
        if run is None:
            pool.extend(ints(seqs), ints(st))
            y = block(ctx, cache, weights, x, ints(seqs), ints(st), heads, group, dim)
        else:
            y = run(x)
        ctx.check_sync()
        assert po.extend(seqs, rows)
        # teacher forcing: the oracle's cache takes the values the library's projection gave
        qkv = ctx.linear_i8(x, *weights[0])
        qh, kh, vh = (host(t.unflatten(1, (-1, dim))) for t in qkv.split([heads * group * dim, heads * dim, heads * dim], 1))
        co.append(kh, vh, seqs, st)
        same_pool(pool, po)
        same_cache(cache, co)
        mid, tol = np.zeros_like(qh), np.zeros(qh.shape)
        for i, s in enumerate(seqs):
            a, b = st[i], st[i + 1]
            mid[a:b], tol[a:b] = attention_bound(qh[a:b], *co.values(s), dim ** -0.5, True, 0, dtype)
        # the second layer's codes move by at most what its input moves: half a step of the grid and the error
        qx, sx = so.quantize_tokens(mid.reshape(len(mid), -1))
        want = so.linear(qx, sx, np_weights[1][0], np_weights[1][1])
        w_abs = np.abs(np_weights[1][0]).astype(np.float64) * np_weights[1][1][:, None]
        slack = (tol.reshape(len(mid), -1) * 2.01 + 1.01 * sx[:, None]) @ w_abs.T
        assert (np.abs(host(y) - want) <= slack + half_step(dtype) * np.abs(want) + 1e-6).all()

    step([0, 1], [37, 5])
    step([2, 0], [16, 1])
    src, dst = pool.fork(ints([0, 0, 1]), ints([3, 4, 5]))
    cache.copy_pages(src, dst)
    co.copy_pages(*po.fork([0, 0, 1], [3, 4, 5]))
    step([0, 3, 4, 5], [1, 1, 1, 1])
    # one captured step, replayed while lengths and pages change
    seqs = [5, 3, 1]
    sd, xs = ints(seqs), torch.zeros((3, hidden), dtype=dtype, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pool.extend(sd)
        ys = block(ctx, cache, weights, xs, sd, None, heads, group, dim)

    def replay(x):
        xs.copy_(x)
        graph.replay()
        return ys.clone()

    for _ in range(18):                            # past the end of a page
        step(seqs, [1, 1, 1], replay)
    pool.free(ints([0, 1]))
    po.free([0, 1])
    where = pool.compact()
    cache.copy_pages(None, where)
    co.copy_pages(None, po.compact())
    step([3, 4, 2], [1, 20, 3])


def test_calls_on_other_streams_and_two_at_once(ctx):
    """Two streams work on caches and workspaces of their own at the same time."""
    rng = np.random.default_rng(29)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    sets = []
    for _ in sides:
        pool, cache, po, co = make(ctx, 300, 64, 4, 70, 4, 128)
        steps(ctx, pool, cache, po, co, [0, 1, 2], [4000, 30, 700], torch.bfloat16, rng)
        q = dev(rng.standard_normal((3, 16, 128)).astype(np.float32), torch.bfloat16)
        w = code_weights(rng, 512, 2048)
        sets.append((cache, q, w, cache.attention(q, ints([0, 1, 2])), ctx.linear_i8(q.flatten(1), *w)))
    seqs = ints([0, 1, 2])
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for side, (cache, q, w, _, _) in zip(sides, sets):
            got.append((cache.attention(q, seqs, stream=side), ctx.linear_i8(q.flatten(1), *w, stream=side)))
        torch.cuda.synchronize()
        for (a, b), (_, _, _, want_a, want_b) in zip(got, sets):
            assert torch.equal(a, want_a) and torch.equal(b, want_b)
    ctx.check_sync()
