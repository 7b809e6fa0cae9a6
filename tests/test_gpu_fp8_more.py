"""GPU tests of the layers in 8-bit floating point: waits that give up, streams, the logistic function."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2511_19438_b200 import build as libbuild
    libbuild.build()
    from paper_2511_19438_b200 import binding as B


@pytest.mark.parametrize("ctas", [1, 2, 4, 8])
def test_a_wait_that_gave_up_keeps_the_whole_cluster_from_storing(ctas):
    """Each CTA of the few-row kernel adds parts of all of its cluster: if one has none, no row is stored."""
    assert B.gptq_check_status() == B.GPTQ_OK
    for who in (-1, 0, ctas - 1):
        stored = torch.zeros(ctas, dtype=torch.int32, device="cuda")
        B.check(B.gptq_selftest_give_up(ctas, who, 200, stored), "selftest launch")      # 200 microseconds
        assert B.gptq_check_status() == (B.GPTQ_OK if who < 0 else B.GPTQ_ERR_TIMEOUT)
        assert (stored == (1 if who < 0 else 0)).all()
    assert B.gptq_check_status() == B.GPTQ_OK
