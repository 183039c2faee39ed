"""Models with an attention in front of a layer: keys and values pass through the 8-bit cache in every forward (calibration,
evaluation, searches, noise), against the oracle's cache and attention in 64 bits."""
import numpy as np
import pytest
import torch

import qcfg_workloads as wl
from oracle import qcfg_oracle as orc
from oracle import serve_oracle as so
from test_gpu_serve import attention_bound

pytestmark = pytest.mark.gpu


def stack(rng, hidden, q_heads, kv_heads, dim, blocks=1):
    """Blocks of q, k, v, o (+ shortcut), ff1, ff2 (+ shortcut); o reads q, which the attention makes its queries."""
    layers, prev = [], -1
    for i in range(blocks):
        at = len(layers)
        L = lambda name, n, k, src, **kw: layers.append(wl.Layer(f"{i}.{name}", n, k, src=src, **kw))
        L("q", q_heads * dim, hidden, prev)
        L("k", kv_heads * dim, hidden, prev)
        L("v", kv_heads * dim, hidden, prev)
        L("o", hidden, q_heads * dim, at, residual_from=prev)
        L("ff1", 2 * hidden, hidden, at + 3, act=wl.ACT_GELU_TANH)
        L("ff2", hidden, 2 * hidden, at + 4, residual_from=at + 3)
        prev = at + 5
    weights = [(rng.standard_normal((l.n_out, l.k_in)) / np.sqrt(l.k_in)).astype(np.float32) for l in layers]
    return layers, weights


class Built:
    def __init__(self, q, seed, m, hidden, q_heads, kv_heads, dim, blocks, **attention):
        rng = np.random.default_rng(seed)
        self.ctx = q.Context(0)
        self.layers, w = stack(rng, hidden, q_heads, kv_heads, dim, blocks)
        self.m, self.n = m, len(self.layers)
        self.weights = [torch.from_numpy(a).cuda() for a in w]
        self.x = torch.from_numpy(rng.standard_normal((m, hidden)).astype(np.float32) * 2).cuda()
        self.model = q.Model(self.ctx, self.layers, self.weights)
        for b in range(blocks):
            self.model.set_attention(6 * b + 3, 6 * b + 1, 6 * b + 2, q_heads, kv_heads, **attention)

    def outputs(self, shift=0):
        """One tensor for every layer's output, `shift` elements behind a 16-byte boundary."""
        out = []
        for l in self.layers:
            flat = torch.full((self.m * l.n_out + shift,), 7.0, device="cuda")
            out.append(flat[shift:].view(self.m, l.n_out))
        return out

    def eval(self, bits, ys):
        self.model.eval_config(bits, self.x, self.m, ys)
        self.ctx.check_sync()

    def close(self):
        self.model.close()
        self.ctx.close()


def expected(ys, at, q_heads, kv_heads, dim, seq_len, page, causal, window, scale):
    """Attention over what layers at, at + 1 and at + 2 gave, and its |error|."""
    q, k, v = (ys[at + j].double().cpu().numpy().astype(np.float32) for j in range(3))
    rows = len(q)
    runs = [(lo, min(lo + seq_len, rows)) for lo in range(0, rows, seq_len)]
    per = -(-min(seq_len, rows) // page)
    pool = so.Pool(len(runs) * per, page, len(runs), per)
    for s, (lo, hi) in enumerate(runs):
        pool.lens[s] = hi - lo
        pool.table[s] = [s * per + j for j in range(pool.pages_for(hi - lo))]
    cache = so.Cache(pool, kv_heads, dim)
    cache.append(k.reshape(rows, kv_heads, dim), v.reshape(rows, kv_heads, dim), list(range(len(runs))), [lo for lo, _ in runs] + [rows])
    out, tol = np.zeros((rows, q_heads, dim)), np.zeros((rows, q_heads, dim))
    for s, (lo, hi) in enumerate(runs):
        kk, vv = cache.values(s)
        out[lo:hi], tol[lo:hi] = attention_bound(q[lo:hi].reshape(-1, q_heads, dim), kk, vv, scale, causal, window, torch.float32)
    return out.reshape(rows, -1), tol.reshape(rows, -1)


SHAPES = [(50, 96, 3, 1, 32, 17, 16, True, 0), (384, 128, 2, 2, 64, 128, 64, False, 0), (200, 64, 4, 2, 16, 100, 32, True, 24),
          (33, 64, 1, 1, 80, 1000, 16, True, 0), (6, 64, 2, 1, 128, 1, 128, True, 0)]


@pytest.mark.parametrize("m,hidden,q_heads,kv_heads,dim,seq_len,page,causal,window", SHAPES)
@pytest.mark.parametrize("shift", [0, 1])
def test_a_layer_behind_an_attention_reads_what_the_oracle_says(m, hidden, q_heads, kv_heads, dim, seq_len, page, causal, window, shift):
    import paper_2302_01382_b200 as q
    scale = 1.3 * dim ** -0.5
    b = Built(q, 3, m, hidden, q_heads, kv_heads, dim, 2, seq_len=seq_len, page_tokens=page, sm_scale=scale, causal=causal, window=window)
    try:
        b.model.calibrate_model(b.x, m)
        act = b.model.act_absmax()
        ys = b.outputs(shift)
        b.eval([16] * b.n, ys)
        for at in (0, 6):                       # the calibration is that forward
            want, tol = expected(ys, at, q_heads, kv_heads, dim, seq_len, page, causal, window, scale)
            top = np.abs(want).max()
            assert abs(act[at + 3] - top) <= tol.max() + 2.0 ** -24 * top
        bits = [8, 16, 8, 8, 4, 16] + [16, 8, 4, 6, 8, 8]
        b.eval(bits, ys)
        for at in (0, 6):
            want, tol = expected(ys, at, q_heads, kv_heads, dim, seq_len, page, causal, window, scale)
            qx = torch.empty((m, q_heads * dim), dtype=torch.int8, device="cuda")
            acc = torch.empty((m, hidden), dtype=torch.int32, device="cuda")
            qw = torch.empty((hidden, q_heads * dim), dtype=torch.int8, device="cuda")
            b.model.debug_dump(at + 3, qx, qw, acc)
            b.ctx.check_sync()
            sx, inv, sw, _ = b.model.scales(at + 3, bits[at + 3])
            qmax = 2 ** (bits[at + 3] - 1) - 1
            # a code is the product in fp32 (half a step of up to qmax), rounded (half a code)
            off = np.abs(qx.cpu().numpy() - np.clip(want * inv, -qmax, qmax))
            assert (off <= 0.5 + tol * inv + qmax * 2.0 ** -24).all(), float((off - tol * inv).max())
            exact = qx.cpu().numpy().astype(np.int64) @ qw.cpu().numpy().astype(np.int64).T
            assert (acc.cpu().numpy() == exact).all()
            # one product, one sum with the shortcut: each half a step of fp32
            y = exact * (np.float32(sx) * np.array(sw, np.float32)).astype(np.float64)[None, :]
            size = np.abs(y)
            if at:
                short = ys[at - 1].double().cpu().numpy()
                y, size = y + short, size + np.abs(short)
            assert (np.abs(ys[at + 3].double().cpu().numpy() - y) <= 2.0 ** -23 * size).all()
    finally:
        b.close()


@pytest.mark.parametrize("grouping,chains", [(True, True), (False, False)])
def test_reuse_is_bit_identical_with_attention(grouping, chains):
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(5)
    b = Built(q, 4, 256, 128, 4, 2, 32, 3, seq_len=64, page_tokens=16)
    try:
        b.ctx.set_grouping(grouping)
        b.ctx.set_gemm_chains(chains)
        b.model.calibrate_model(b.x, b.m)
        order = [int(i) for i in rng.permutation(b.n)]
        seq = wl.greedy_sequence(order, rng.random(b.n) < 0.5)[:24] + [rng.choice(np.array([4, 8, 16], np.uint8), size=b.n) for _ in range(8)]
        seq += [seq[-1], seq[-1]]
        taps = [[int(l) for l in rng.choice(b.n, size=int(rng.integers(0, 4)), replace=False)] for _ in seq]
        runs, launches = [], []
        for reuse in (False, True):
            b.ctx.set_prefix_reuse(reuse)
            ys, got, start = b.outputs(), [], b.ctx.launch_count()
            for bits, tap in zip(seq, taps):
                b.eval(bits, [y if l == b.n - 1 or l in tap else None for l, y in enumerate(ys)])
                got.append([ys[l].clone() for l in [b.n - 1] + tap])
            launches.append(b.ctx.launch_count() - start)
            runs.append(got)
        for i, (a, c) in enumerate(zip(*runs)):
            assert all(torch.equal(s, t) for s, t in zip(a, c)), i
        assert launches[1] < launches[0]
    finally:
        b.close()


def test_searches_and_noise_go_through_the_attention():
    import paper_2302_01382_b200 as q
    b = Built(q, 6, 128, 64, 2, 1, 32, 2, seq_len=48, page_tokens=16)
    try:
        b.model.calibrate_model(b.x, b.m)
        ys = b.outputs()
        last = [None] * (b.n - 1) + [ys[-1]]
        b.eval([16] * b.n, last)
        ref = ys[-1].double().clone()
        for algorithm in (0, 1):
            bits, visited, fidelity, count = b.model.search(algorithm, list(range(b.n)), [16, 8, 4], 0.97, b.x, b.m)
            assert count == len(visited)
            for cfg, f in zip(visited, fidelity):
                b.eval(cfg, last)
                want = 1 - float((ys[-1].double() - ref).norm() / ref.norm())
                assert abs(f - want) <= 1e-12
        noises = [torch.from_numpy(a).cuda() for a in wl.standard_normal_like([w.cpu().numpy() for w in b.weights], 9)]
        together = b.model.noise_sensitivity(b.x, b.m, noises, 0.05)
        for l in range(b.n):
            alone = b.model.noise_sensitivity(b.x, b.m, [t if i == l else None for i, t in enumerate(noises)], 0.05)
            assert alone[l] == together[l] and alone[l] > 0
        table = b.model.latency_table(b.x, b.m, [8, 16], 2)
        assert all(t > 0 for row in table for t in row)
    finally:
        b.close()


def test_attention_follows_the_number_of_rows():
    """The cache is laid out anew when the rows change, and back."""
    import paper_2302_01382_b200 as q
    b = Built(q, 7, 100, 64, 2, 2, 32, 1, seq_len=40, page_tokens=16)
    try:
        b.model.calibrate_model(b.x, b.m)
        bits = [8] * b.n
        first = {}
        for m in (100, 37, 100, 80, 37):
            y = torch.empty((m, 64), device="cuda")
            b.model.eval_config(bits, b.x, m, [None] * (b.n - 1) + [y])
            b.ctx.check_sync()
            assert torch.equal(y, first.setdefault(m, y.clone()))
        # whole sequences do not see one another, so they give the same whatever comes behind them
        assert torch.equal(first[80], first[100][:80])
    finally:
        b.close()


def test_attention_refusals():
    import paper_2302_01382_b200 as q
    rng = np.random.default_rng(1)
    ctx = q.Context(0)
    try:
        layers, w = stack(rng, 64, 4, 2, 16)
        weights = [torch.from_numpy(a).cuda() for a in w]
        model = q.Model(ctx, layers, weights)
        x = torch.from_numpy(rng.standard_normal((32, 64)).astype(np.float32)).cuda()
        model.calibrate_model(x, 32)
        good = dict(layer=3, k_layer=1, v_layer=2, q_heads=4, kv_heads=2, seq_len=16, page_tokens=16)
        for change, error in ((dict(layer=6), "EINVAL"), (dict(layer=-1), "EINVAL"), (dict(k_layer=3), "EINVAL"), (dict(v_layer=-1), "EINVAL"),
                              (dict(layer=0), "EINVAL"), (dict(q_heads=3), "ESHAPE"), (dict(q_heads=0), "ESHAPE"), (dict(kv_heads=3), "ESHAPE"),
                              (dict(kv_heads=4), "ESHAPE"), (dict(q_heads=8, kv_heads=4), "ESHAPE"), (dict(v_layer=0), "ESHAPE"),
                              (dict(page_tokens=48), "ESHAPE"), (dict(seq_len=0), "ESHAPE"), (dict(sm_scale=0.0), "EINVAL"),
                              (dict(sm_scale=float("nan")), "EINVAL"), (dict(window=-1), "EINVAL"), (dict(window=4, causal=False), "EINVAL")):
            with pytest.raises(q.QcfgError, match=error):
                model.set_attention(**{**good, **change})
        model.eval_config([8] * 6, x, 32)           # a refusal changes nothing
        model.set_attention(**good)
        with pytest.raises(q.QcfgError, match="ESTATE"):
            model.set_attention(**good)
        with pytest.raises(q.QcfgError, match="ESTATE"):
            model.eval_config([8] * 6, x, 32)       # the maxima are another model's
        model.calibrate_model(x, 32)
        model.eval_config([8] * 6, x, 32)
        with pytest.raises(q.QcfgError, match="ESHAPE"):
            model.adjust_scales([8] * 6, x, 32, 1)
        ctx.check_sync()
        model.close()
    finally:
        ctx.close()
