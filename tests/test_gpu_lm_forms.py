"""Every form that sizes alone choose for the operators around a model's matrices, each against its formula in 64 bits.  That these sizes
reach all forms is checked without a GPU (test_lm_shape)."""
import pytest
import torch

from test_gpu_lm import DEV, TYPES, check_xent, near, q8_want, randn, same, scd, weights8, xent_inputs  # noqa: F401  (scd: the fixture)

pytestmark = pytest.mark.gpu

XENT_16 = [(1, 520, 8), (1, 520, 20001), (64, 2056, 4100), (65, 520, 20001), (1, 2056, 8), (65, 1001, 8), (1, 4096, 20001), (4001, 4099, 8), (1, 1001, 2049),
           (1000, 8, 2003), (2300, 8, 32001), (200, 520, 20001), (2300, 520, 32001), (65, 4099, 20001), (33, 2056, 8), (1, 4099, 2049), (33, 1001, 2049),
           (33, 2048, 2049), (33, 4099, 2049), (2050, 4099, 4100), (2300, 1001, 32001), (130, 2048, 32001), (4001, 520, 20001), (513, 1001, 20001),
           (4001, 1544, 20001), (16003, 4096, 200), (16003, 136, 4100), (1000, 520, 70000)]
XENT_32 = [(2300, 8, 32001), (1, 256, 8), (1, 256, 65), (2900, 8, 1030), (1, 1544, 32001), (65, 256, 20001), (1, 2056, 8), (1, 2056, 65), (33, 4099, 8),
           (33, 4099, 65), (2900, 1001, 130), (4001, 256, 1030), (33, 2056, 32001), (1, 8, 2049), (33, 8, 2049), (1, 2056, 2049), (2900, 9, 32001),
           (2300, 64, 32001), (2300, 72, 32001), (1, 9, 8), (1, 9, 2049), (33, 9, 2049), (1, 1001, 2049), (65, 9, 32001), (1, 1001, 32001), (200, 9, 32001),
           (33, 1000, 2049), (33, 1001, 2049), (33, 1001, 20001), (65, 1001, 20001), (200, 1001, 20001), (2300, 1001, 32001), (4001, 129, 20001), (9000, 1, 8199),
           (9000, 1001, 1), (1, 4099, 70000), (33, 4099, 70000), (65, 4099, 70000), (1000, 256, 70000)]
XENT = [(torch.bfloat16, *s) for s in XENT_16] + [(torch.float16, *s) for s in XENT_16] + [(torch.float32, *s) for s in XENT_32]
Q8 = [(1, 264, 193), (2, 1000, 200), (3, 1000, 200), (9, 1000, 200), (4, 40000, 100), (16, 14336, 193), (33, 2000, 1501), (64, 14336, 200), (129, 1032, 14336),
      (333, 2000, 1501), (2300, 4096, 6000), (2300, 1000, 6004)]


@pytest.mark.parametrize("dtype,N,D,V", XENT, ids=[f"{str(t)[6:]}-{n}-{d}-{v}" for t, n, d, v in XENT])
def test_xent_in_every_form(scd, dtype, N, D, V):  # noqa: F811
    x, w, t, g = xent_inputs(N, D, V, dtype, 400, ignored=0.0 if N == 1 else 0.2)
    # targets at both ends of the vocabulary and of pieces of it
    ends = torch.tensor([V - 1, 0, V // 2 // 256 * 256, V // 256 * 256, max(V // 256 * 256 - 1, 0), min(255, V - 1)], device=DEV)
    t[:len(ends)] = ends[:min(N, len(ends))].clamp(max=V - 1)
    check_xent(scd, x, w, t, g, scale=0.9)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", Q8)
def test_q8_linear_in_every_form(scd, dtype, M, K, N):  # noqa: F811
    x = randn((M, K), 410, dtype)
    wq, ws = weights8(N, K, 411)
    bias = randn((N,), 412, dtype)
    y = scd.scd_q8_linear(x, wq, ws, bias=bias)
    q, s = scd.scd_q8_rows(x)
    near(y, *q8_want(q, s, wq, ws, bias, dtype))
    same(y, scd.scd_q8_matmul(q, s, wq, ws, K, dtype=dtype, bias=bias))
