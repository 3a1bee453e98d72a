"""Cross entropy where digits are easily lost: tokens whose target is all but certain, weights of very different size, entries at the
ends of the range.  Inputs are chosen so that logits are exact in f32; bounds follow from the roundings that remain.  E, U as in test_gpu_lm."""
import pytest
import torch

from test_gpu_lm import DEV, E, TYPES, U, check_xent, near, off_by_one, same, scd, xent_inputs  # noqa: F401  (scd: the fixture)

pytestmark = pytest.mark.gpu


def confident(N, V, dtype):
    """Token n has logit 0 for its target n and -c_n for the others, c_n = 12 .. 20 in eighths: 1 - p is V exp(-c_n)."""
    c = 12.0 + (torch.arange(N, device=DEV) % 64) / 8.0
    x = torch.diag(c).to(dtype)
    w = torch.full((V, N), -1.0, device=DEV)
    w[:N].fill_diagonal_(0.0)
    return c.double(), x, w.to(dtype), torch.arange(N, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(64, 64), (64, 2500), (200, 700)])
def test_weight_gradient_of_confident_tokens(scd, dtype, N, V):  # noqa: F811
    c, x, w, t = confident(N, V, dtype)
    g = torch.full((N,), 0.375, device=DEV)
    _, lse = scd.scd_xent(x, w, t)
    _, dW = scd.scd_xent_grad(x, w, t, lse, g, want_dX=False)
    # entry (n, n) of dW is one term, g (p_n - 1) c_n with p_n = exp(-lse_n); p is off by two steps of f32 below 1, dz has at
    # least the type's digits, and so has the result
    want = 0.375 * torch.expm1(-lse.double()) * c
    near(dW[:N].diagonal(), want, 0.375 * c * 2 * E + 2.02 * U[dtype] * want.abs() + 4 * E * want.abs())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V,shift", [(64, 64, 0), (64, 2500, 200), (300, 700, 200), (3, 40000, 200)])
def test_losses_of_confident_tokens(scd, dtype, N, V, shift):  # noqa: F811
    """The target's logit is the largest: the loss is log(1 + the others' exponentials), whatever the logit itself is."""
    c, x, w, t = confident(N, V, dtype)
    x = torch.cat([x, torch.ones((N, 1), dtype=dtype, device=DEV)], 1)
    w = torch.cat([w, torch.full((V, 1), float(shift), device=DEV).to(dtype)], 1)  # adds `shift` to every logit, exactly
    loss, lse = scd.scd_xent(x, w, t)
    others = (V - 1) * torch.exp(-c)
    want = torch.log1p(others)
    # a lane adds at most 32 exponentials in f32, two more sums and a product follow, the rest is in 64 bits: 35 roundings of a sum
    # that holds the target's 1; the others' exponents are up to 20 log2 e = 29, off by half a step each
    tol = 36 * E + 60 * E * others
    near(loss, want, tol + E * want)
    near(lse, want + shift, tol + E * (want + shift))


@pytest.mark.parametrize("N", [20, 70, 300])
def test_f16_gradients_of_tokens_of_little_weight(scd, N):  # noqa: F811
    """Rows of W are unit vectors, so that dX is dz itself; all tokens but one weigh 2^-27 of that one."""
    V = 72
    x = torch.randn((N, V), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).half()
    w, t = torch.eye(V, device=DEV).half(), torch.arange(N, device=DEV) % V
    ref = 2.0 ** 15
    g = ref * 2.0 ** -27 * (1.0 + torch.rand(N, generator=torch.Generator(device=DEV).manual_seed(6), device=DEV))
    g[0] = ref
    _, lse = scd.scd_xent(x, w, t)
    dX, _ = scd.scd_xent_grad(x, w, t, lse, g, want_dW=False)
    p = (x.double() - lse.double()[:, None]).exp()
    want = g.double()[:, None] * (p - torch.nn.functional.one_hot(t, V).double())
    # p: exponents below 16, two steps of it; dz: the type's digits, or steps of 2^-24 of numbers up to 2^15; the result: its digits or steps
    tol = g.double()[:, None] * 24 * E + 2.02 * U[torch.float16] * want.abs() + 2.0 ** -39 * ref + 2.0 ** -25
    near(dX, want, tol)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [20, 70])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_weight_that_is_not_finite_stays_with_its_token(scd, dtype, N, bad):  # noqa: F811
    V, D = 72, 64
    gen = torch.Generator(device=DEV).manual_seed(7)
    x, w = (torch.randn((n, D), generator=gen, device=DEV).to(dtype) for n in (N, V))
    t = torch.arange(N, device=DEV) % V
    g = 100.0 + 200.0 * torch.rand(N, generator=gen, device=DEV)
    _, lse = scd.scd_xent(x, w, t)
    g[3] = 0.0
    want, _ = scd.scd_xent_grad(x, w, t, lse, g, want_dW=False)
    g[3] = bad
    got, _ = scd.scd_xent_grad(x, w, t, lse, g, want_dW=False)
    rest = torch.arange(N, device=DEV) != 3
    assert not torch.isfinite(got[3]).any() and torch.isfinite(want).all()
    same(got[rest], want[rest])  # (held relative to the largest finite weight)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V", [(7, 72, 300), (300, 72, 300), (40, 256, 2500), (600, 1030, 700)])
def test_gradients_with_very_large_entries(scd, dtype, N, D, V):  # noqa: F811
    """Entries just below the 2^100 that the header names, in one column of X, and in another of W, where the other matrix is zero."""
    x, w, t, g = xent_inputs(N, D, V, dtype, 300, ignored=0.1)
    x[:, 1] = x[:, 1].clamp(-1, 1) * 2.0 ** 99
    w[:, 1] = 0
    w[:, 2] = w[:, 2].clamp(-1, 1) * 2.0 ** 99
    x[:, 2] = 0
    check_xent(scd, x, w, t, g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D,V", [(5, 264, 530), (150, 264, 530), (300, 520, 4097)])
def test_gradients_do_not_depend_on_where_the_hidden_states_lie(scd, dtype, N, D, V):  # noqa: F811
    x, w, t, g = xent_inputs(N, D, V, dtype, 310)
    _, lse = scd.scd_xent(x, w, t)
    for a, b in zip(scd.scd_xent_grad(off_by_one(x), w, t, lse, g), scd.scd_xent_grad(x, w, t, lse, g)):
        same(a, b)
