"""Products in 8-bit floating point and the gated block in every form of the kernels, with odd sizes, their types and both activations.  Tolerances are
those of test_gpu_f8.py."""
import pytest

pytest.importorskip("torch")
import f8_sizes  # noqa: E402
from test_gpu_f8 import test_gated as check_gated  # noqa: E402
from test_gpu_f8_forms import test_products as check_products  # noqa: E402

pytestmark = pytest.mark.gpu
PRODUCTS = [size for sizes in f8_sizes.PRODUCTS.values() for size in sizes]
GATED = [size for sizes in f8_sizes.GATED.values() for size in sizes]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product_in_every_form(m, n, k):
    check_products(m, n, k)


@pytest.mark.parametrize("act,dtype", [(0, "bf16"), (1, "bf16"), (1, "f32"), (0, "f16")])
@pytest.mark.parametrize("m,f,k", GATED)
def test_gated_in_every_form(m, f, k, act, dtype):
    check_gated(m, f, k, dtype, act)
