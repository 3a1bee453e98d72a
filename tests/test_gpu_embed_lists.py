"""The embedding's gradient where a token's list meets the edges that its sum is cut at."""
import pytest
import torch

from test_gpu_lm import DEV, check_embed_grad, gen, randn, scd  # noqa: F401  (scd: the fixture)

pytestmark = pytest.mark.gpu

# Lists of the sorted order are cut into pieces of 16 places: lists of 15 to 17 and 31 to 33 tokens, beginning and ending on, before and behind
# a piece's first place, neighbours that share a piece, and longer ones that are summed in 16 stretches.
LISTS = [[15, 16, 17, 31, 32, 33] * 3, [16] * 20, [17] * 17, [32] * 9, [15, 17] * 9, [1, 16, 31, 17, 32, 15, 33, 160], [20, 20, 300], [8, 300, 8, 16, 1],
         [0, 16, 0, 17, 240, 0], [257], [256, 1], [1, 256], [272, 33, 255, 257, 513, 1], [4096, 16, 4111, 17]]


@pytest.mark.parametrize("dtype,D", [(torch.float32, 24), (torch.float32, 23), (torch.bfloat16, 1032), (torch.float16, 3)])
@pytest.mark.parametrize("lists", LISTS, ids=[str(i) for i in range(len(LISTS))])
def test_embed_grad_lists_around_the_length_of_a_piece(scd, lists, dtype, D):  # noqa: F811
    V = len(lists)
    assert sum(lists) > 256  # (up to 256 tokens are summed without a sort)
    tokens = torch.repeat_interleave(torch.arange(V, device=DEV), torch.tensor(lists, device=DEV))
    tokens = tokens[torch.randperm(tokens.numel(), generator=gen(420), device=DEV)]
    check_embed_grad(scd, tokens, randn((tokens.numel(), D), 421, dtype), V, -1, 1.0)


@pytest.mark.parametrize("dtype,D", [(torch.float32, 24), (torch.bfloat16, 1031)])
@pytest.mark.parametrize("lists", [[15, 16, 17, 31, 32, 33], [255], [256], [255, 1], [0, 100, 0, 156], [1] * 256, [64, 65, 63, 64]], ids=str)
def test_embed_grad_lists_of_few_tokens(scd, lists, dtype, D):  # noqa: F811
    V = len(lists)
    tokens = torch.repeat_interleave(torch.arange(V, device=DEV), torch.tensor(lists, device=DEV))
    tokens = tokens[torch.randperm(tokens.numel(), generator=gen(422), device=DEV)]
    check_embed_grad(scd, tokens, randn((tokens.numel(), D), 423, dtype), V, -1, 1.0)
