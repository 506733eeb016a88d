"""GPU: matrices of more rows than the C interface counts are refused, not taken for the rest modulo 2^32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_more_rows_than_32_bits_count():
    from paper_2405_14917_b200 import binding as slim
    M = 2 ** 32 + 5
    s = torch.empty(M, 1, dtype=torch.float16, device="cuda")
    index, value = torch.zeros(1, 1, dtype=torch.int32, device="cuda").expand(M, 1), torch.zeros(1, 1, device="cuda").expand(M, 1)
    with pytest.raises(ValueError, match="rows"):
        slim._rows(s, "logits", (torch.float16,))
    with pytest.raises(ValueError, match="rows"):
        slim.distill_loss(s, index, value)
    with pytest.raises(ValueError, match="rows"):
        slim.fp8_quantize(torch.empty(M, 0, dtype=torch.float16, device="cuda"))
