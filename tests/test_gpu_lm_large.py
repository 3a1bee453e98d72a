"""The operators around a model's matrices at their largest: row counts at the end of what the header allows."""
import pytest
import torch

from test_gpu_lm import DEV, gen, scd  # noqa: F401  (scd: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("short", [0, 16384, 40000])
def test_embed_grad_of_as_many_tokens_as_there_may_be(scd, short):  # noqa: F811
    """2^31 - 1 tokens all of which count, and a little fewer: places of the sorted order and of pieces that pass 32 bits."""
    N, V = 2 ** 31 - 1 - short, 1000
    tokens = torch.randint(0, V, (N,), generator=gen(1), device=DEV, dtype=torch.int32)
    dY = torch.zeros((N, 1), dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 1, 2 ** 30, N // 3, N - 16385, N - 17, N - 2, N - 1], device=DEV)
    tokens[N - 1], tokens[N - 2] = V - 1, V - 1  # the last places of the order
    dY[at, 0] = torch.arange(1, 9, device=DEV).to(torch.bfloat16)
    want = torch.zeros(V, dtype=torch.float64, device=DEV).index_add_(0, tokens[at].long(), torch.arange(1, 9, device=DEV).double())
    got = scd.scd_embed_grad(tokens, dY, V)
    assert torch.equal(got[:, 0].double(), want)
