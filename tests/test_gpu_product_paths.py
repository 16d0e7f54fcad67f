"""Projections and gated blocks on the GPU against the float64 oracle at shapes that reach every way of cutting a product;
test_product_plan checks on the CPU that they do. Tolerances: those of test_gpu_product."""
import pytest

from test_gpu_product import run
from test_product_plan import GRADIENTS, PATHS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,F,glu", PATHS)
def test_forward(M, K, F, glu):
    run(1, M, K, F, "bf16", "silu", bias=True, glu=glu, train=False, **({} if glu else dict(gate="shared", residual=True)))


@pytest.mark.parametrize("M,K,F,glu", GRADIENTS)
def test_gradients(M, K, F, glu):
    run(1, M, K, F, "bf16", "silu", bias=True, glu=glu)


@pytest.mark.parametrize("M,K,F,glu", GRADIENTS[2:])
def test_gradients_of_plain_projections(M, K, F, glu):
    """Nothing between dY and dZ (a gated block in fp16)."""
    run(1, M, K, F, "fp16", "silu" if glu else "none", glu=glu)


@pytest.mark.parametrize("B,N,K,F,glu", [(1, 1, 20000, 40, False), (4, 1, 12000, 130, False), (2, 3, 6000, 100, True), (16, 1, 8200, 16, True)])
def test_few_tokens_of_long_rows(B, N, K, F, glu):
    run(B, N, K, F, "bf16", "gelu", bias=True, glu=glu, **({} if glu else dict(gate="adaptive", residual=True)))
