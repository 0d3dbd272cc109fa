"""The gated feed-forward block on the GPU where its variants meet: few tokens and one output, and sums of many terms of one sign."""
import pytest
import torch

from test_feed_forward_gpu import _check

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    from paper_2004_05298_b200 import binding
    yield binding
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["rows", "padded", "off"])
def test_few_tokens_and_one_output(B, dtype, layout):
    """w_down has one row, whose length need not be a multiple of 16 bytes for it to be read in place."""
    for T in (1, 2, 32, 33):
        for C, F in ((64, 65), (64, 1), (72, 200), (65, 66), (8, 4097)):
            _check(B, T, C, F, 1, dtype, T, layout, train=False)
            _check(B, T, C, F, 1, dtype, T, layout)
