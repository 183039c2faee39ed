"""What qcfg_gemm_i8_requant writes behind an output's last column."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n", [(5, 1), (100, 51), (300, 1001), (3000, 2311), (129, 64)])
@pytest.mark.parametrize("bits", [8, 16])
def test_requant_zeroes_the_last_16_bytes_and_nothing_else(m, n, bits):
    import paper_2302_01382_b200 as q
    c = q.Context(0)
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n)
    x, w = (torch.randint(-127, 128, (r, 256), generator=g, device="cuda", dtype=torch.int8) for r in (m, n))
    dtype = torch.int8 if bits == 8 else torch.bfloat16
    out = torch.full((m + 2, (n + 15) // 16 * 16 + 32), 9, dtype=dtype, device="cuda")
    c.gemm_i8_requant(x, w, 256, 0.01, torch.rand(n, generator=g, device="cuda"), q.ACT_NONE, 0.1, bits, out=out[1:m + 1])
    c.check_sync()
    each = 16 // out.element_size()
    end = (n + each - 1) // each * each
    assert not out[1:m + 1, n:end].any()
    out[1:m + 1, :end] = 9
    assert (out == 9).all()
    c.close()
