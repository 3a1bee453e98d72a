"""Arrays that ask torch for a gradient: the operators around a model's matrices refuse them rather than drop it."""
import pytest
import torch

from test_gpu_lm import DEV, same, scd, weights8, xent_inputs  # noqa: F401  (scd: the fixture)

pytestmark = pytest.mark.gpu


def test_arrays_that_ask_for_a_gradient_are_refused_while_torch_records(scd):  # noqa: F811
    x, w, t, g = xent_inputs(5, 64, 40, torch.float32, 500, ignored=0.0)
    wq, ws = weights8(16, 64, 501)
    bias = torch.zeros(16, device=DEV)
    loss, lse = scd.scd_xent(x, w, t)
    q, s = scd.scd_q8_rows(x)
    calls = [  # (the call, the arrays of it that torch could ask a gradient of)
        (lambda E: scd.scd_embed(E, t), [w]),
        (lambda dY: scd.scd_embed_grad(t, dY, 40), [x]),
        (lambda X, s, b: scd.scd_q8_linear(X, wq, s, bias=b), [x, ws, bias]),
        (lambda r, s, b: scd.scd_q8_matmul(q, r, wq, s, 64, dtype=torch.float32, bias=b), [s, ws, bias]),
        (lambda X, W: scd.scd_xent(X, W, t)[0], [x, w]),
        (lambda X, W, l, v: scd.scd_xent_grad(X, W, t, l, v)[0], [x, w, lse, g]),
    ]
    for call, arrays in calls:
        want = call(*arrays)
        for i in range(len(arrays)):
            asking = [a.clone().requires_grad_(i == j) for j, a in enumerate(arrays)]
            with pytest.raises(ValueError, match="autograd"):
                call(*asking)
            with torch.no_grad():
                same(call(*asking), want)
            same(call(*[a.detach() for a in asking]), want)
    same(scd.scd_q8_rows(x.clone().requires_grad_())[0], q)  # (integers: there is no gradient to lose)
