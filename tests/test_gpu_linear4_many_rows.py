"""4-bit products of more rows than a decode batch has: a prompt's.  The tolerance is that of the other products: fp32 sums of n exact products, a scale,
bias and residual, rounded to fp16 once."""
import pytest

from test_gpu_linear4 import product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("m", [257, 320, 511, 1000, 2049, 4095, 4096])
def test_many_rows(m, group, zeros):
    product(m, 144, 640, group, zeros, residual=m % 2 == 0, relu=m % 3 == 0)


@pytest.mark.parametrize("m,n_out,n_in", [(300, 4096, 1024), (1024, 2064, 4096), (4096, 1024, 2048), (600, 48, 16384)])
def test_many_rows_of_larger_products(m, n_out, n_in):
    product(m, n_out, n_in, 128, False, residual=True)
    product(m, n_out, n_in, 64, True, segments=[n_out - 32, 16, 16])
