"""The 8-bit serving operators where they can go wrong: outputs wider than one pass of a kernel, refused calls and what comes behind
them, values of very different sizes, numbers out of range.  Helpers, oracle and the way tolerances are counted: test_gpu_serve.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from test_gpu_serve import ACTS, DTYPES, U, check_attention, code_weights, ctx, dev, half_step, host, ints, linear_bound, make, same_cache, same_pool, starts_of, steps  # noqa: F401
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
