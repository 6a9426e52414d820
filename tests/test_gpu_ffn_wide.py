"""A gated gradient of so many columns that their sums, 64 a workgroup, would take a launch of 2^32 threads."""
import gc

import pytest
import torch

import mm_routes as R
from paper_2309_17224_amd import fp8lin as F
from test_gpu_ffn import word

pytestmark = pytest.mark.gpu


@pytest.fixture
def emptied():
    """The memory of a test of 100 GB given back before and after it."""
    gc.collect()
    torch.cuda.empty_cache()
    yield
    gc.collect()
    torch.cuda.empty_cache()


def test_bias_gradient_and_codes_of_more_columns_than_a_launch_has(gpu, emptied):
    K, N = 1 << 29, 128
    assert R.epilogue(3, 1, K, N)[0] == R.STREAM
    one = torch.ones(1, device=gpu)
    w8 = torch.full((K, N), int(one.to(torch.float8_e4m3fn).view(torch.uint8)), dtype=torch.uint8, device=gpu)
    dy8 = torch.full((1, N), int(one.to(torch.float8_e5m2).view(torch.uint8)), dtype=torch.uint8, device=gpu)
    gu = torch.randint(-2, 3, (1, 2 * K), dtype=torch.int8, device=gpu).to(torch.bfloat16)
    db = torch.empty(2 * K, device=gpu)
    fq = F.FusedQuant(torch.empty((1, 2 * K), dtype=torch.uint8, device=gpu), word(0, gpu),
                      torch.empty(F.fp8_linear_quantise_ws_bytes(1, 2 * K), dtype=torch.uint8, device=gpu), F.E5M2,
                      bias_pred=word(1, gpu), amax_bits=word(0, gpu))
    dgu = F.fp8_linear_bwd_dx_glu(dy8, word(3, gpu), w8, word(4, gpu), gu, F.ACT_NONE, db=db, fq=fq)  # t = 1
    assert torch.equal(dgu[:, :K], gu[:, K:]) and torch.equal(dgu[:, K:], gu[:, :K])
    assert torch.equal(db, dgu[0].float())
    del w8, db, gu
    q, _, bias, amax, _ = F.fp8_quantise(dgu, F.E5M2, 0)
    assert int(fq.bias) == int(bias) and int(fq.amax_bits) == int(amax) and torch.equal(fq.q, q)
