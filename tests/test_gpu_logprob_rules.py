"""What the calls on logits promise beyond their values: rows of more than 2^30 entries, threads without a row."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_logprobs import E, MARK, env  # noqa: E402, F401


def test_gradient_of_a_row_of_more_than_a_billion_entries(env):  # noqa: F811
    """Threads behind the last row, and those of a row behind the count, do nothing: 1.3e9 entries by four chunks 3.2e8 entries apart reach beyond 2^31 from there."""
    sf, ctx = env
    V, k = 1_300_000_003, 2
    x = torch.zeros(2 * V, dtype=torch.bfloat16, device="cuda").view(2, V)
    x[:, 5], x[0, V - 1] = 20.0, 21.0
    n_dev = torch.ones(1, dtype=torch.int32, device="cuda")
    labels, ids = torch.tensor([7, 7], dtype=torch.int32, device="cuda"), torch.tensor([[V - 1, 5], [5, 0]], dtype=torch.int32, device="cuda")
    s = V - 2 + np.exp(20.0) + np.exp(21.0)
    lse = torch.full((2,), float(np.log(s)), device="cuda")
    g, gt = 0.5, (2.0, -1.0)
    d = torch.full_like(x, MARK)
    sf.sf_label_logprobs_backward(ctx, x, labels, lse, d, d_logprob=torch.full((2,), g, device="cuda"), top_ids=ids, d_top_logprobs=torch.tensor([gt, gt], device="cuda"), n_dev=n_dev)
    sf.sf_ctx_poll(ctx)
    total = g + sum(gt)
    p = np.exp([0.0, 20.0, 21.0]) / s
    # lse rounded to fp32 is off by e |lse|, an exponential by (4 + 2 span) e; half a step of bf16 on top
    for i, want in ((7, g - p[0] * total), (5, gt[1] - p[1] * total), (V - 1, gt[0] - p[2] * total), (0, -p[0] * total), (V - 2, -p[0] * total), (V // 2, -p[0] * total)):
        assert abs(float(d[0, i]) - want) <= 2.0 ** -8 * abs(want) + 100 * E * total, i
    rest = d[0].clone()
    rest[torch.tensor([5, 7, V - 1], device="cuda")] = d[0, 0]
    assert bool((rest == d[0, 0]).all()) and bool((d[1] == MARK).all())
