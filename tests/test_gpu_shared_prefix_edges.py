"""Attention over a shared prefix alone, behind few pairs (streamed) and many (tensor cores), one and several tiles of pairs."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cass():
    import paper_2605_26558_b200 as m
    return m


@pytest.mark.parametrize("dtype,how", [(torch.bfloat16, "bphd"), (torch.float16, "bhpd")])
@pytest.mark.parametrize("b,rows,nq,nk,d,prefix", [
    (1, 1, 4, 2, 64, 1), (1, 1, 32, 8, 128, 5000), (9, 1, 32, 8, 128, 4001), (40, 1, 8, 2, 128, 129), (33, 5, 8, 2, 64, 700), (70, 3, 24, 2, 128, 257),
    (150, 1, 4, 2, 64, 128), (24, 1, 8, 2, 96, 300), (5, 16, 16, 1, 64, 4000)])
def test_a_prefix_alone(cass, dtype, how, b, rows, nq, nk, d, prefix):
    from test_gpu_shared_prefix import Case
    Case(b, rows, nq, nk, d, prefix, 0, [0] * b, dtype, how, seed=b).check(cass, weights=False)
