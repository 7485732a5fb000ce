"""C <- beta C where there is nothing to add up, whatever alpha is."""
import pytest

torch = pytest.importorskip("torch")
import paper_2508_03984_amd as oz  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("alpha", [2.0, 0.0, float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("m,n", [(1, 7), (70, 70), (300, 5000)])
def test_no_columns(m, n, alpha):
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        C = torch.full((m, n), 3.0, dtype=dtype, device="cuda")
        oz.oz2_f8_gemm(m, n, 0, alpha, None, None, -0.5, C, n)
        assert (C == -1.5).all()
        C.fill_(float("nan"))
        oz.oz2_f8_gemm(m, n, 0, alpha, None, None, 0.0, C, n)
        assert (C == 0).all()
