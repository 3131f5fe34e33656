"""Pins of the test-side 4-bit reference, and what the 4-bit and expert calls refuse or compute without a GPU."""
import numpy as np
import pytest

import packed_rows as pr


def test_reference_codes_and_ties():
    grid = np.array([0, .25, .2500001, .5, .75, 1.25, 1.75, 2.5, 2.500001, 3.5, 5, 5.0001, 6, 7.9])
    assert pr.nearest_code(grid).tolist() == [0, 0, 1, 1, 2, 2, 4, 4, 5, 6, 6, 7, 7, 7]


def test_reference_scales():
    x = np.zeros((5, 32))
    x[0, 3] = 6.0                       # 2^2 <= 6 < 2^3: scale 1
    x[1, 0] = -1.0                      # scale 2^-2, code of 4 with its sign
    x[2, 5] = 2.0 ** -149               # the scale does not go below 2^-127
    x[3, 1] = np.inf
    code, byte = pr.quantise(x)
    assert byte[:, 0].tolist() == [127, 125, 0, 255, 0]
    assert code[0, 3] == 7 and code[1, 0] == 14 and code[2].sum() == 0 and code[3].sum() == 0
    assert np.isnan(pr.rounded(x)[3]).all() and pr.rounded(x)[1, 0] == -1.0


def test_every_value_of_the_format_is_kept():
    rng = np.random.default_rng(0)
    code = rng.integers(0, 16, (40, 64)).astype(np.uint8)
    code[:, ::32] = 7                   # a block's largest magnitude is a 6, so its scale is found again
    byte = rng.integers(0, 250, (40, 2)).astype(np.uint8)
    x = pr.values(code, byte, 64)
    c, b = pr.quantise(x)
    assert np.array_equal(b, byte) and np.array_equal(pr.values(c, b, 64), x)


@pytest.fixture(scope="module")
def sf():
    from paper_2402_03694_b200 import build, binding
    build.build()
    return binding


def test_sizes(sf):
    for rows, K in ((0, 5), (1, 1), (128, 128), (129, 129), (1000, 4000)):
        assert sf.sf_mx4_sizes(rows, K) == (rows * (-(-K // 32)) * 16, -(-rows // 128) * (-(-K // 128)) * 512)
    for K in (0, (1 << 24) + 1):
        with pytest.raises(sf.SfError) as e:
            sf.sf_mx4_sizes(4, K)
        assert e.value.status == sf.SF_ERR_ARG
    assert sf.sf_expert_sort_workspace(0, 1, 1) == 0
    assert sf.sf_expert_sort_workspace(10, 3, 7) == 28
    for n, k, E in ((1, 1, 0), (1, 1, 1025), (1, 0, 4), (1 << 30, 2, 4), (1, 1025, 4)):
        with pytest.raises(sf.SfError):
            sf.sf_expert_sort_workspace(n, k, E)


def test_host_tensors_and_wrong_shapes_are_refused(sf):
    torch = pytest.importorskip("torch")
    x, u8 = torch.zeros(4, 32), torch.zeros(4096, dtype=torch.uint8)
    i32, f32 = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for call in (lambda: sf.sf_mx4_quantise(None, x, u8, u8), lambda: sf.sf_mx4_unpack(None, u8, u8, x),
                 lambda: sf.sf_mx4_matmul(None, u8, u8, u8, u8, 32, x), lambda: sf.sf_mx4_matmul_experts(None, u8, u8, u8, u8, 32, i32[0], x),
                 lambda: sf.sf_expert_gate(None, x, 0, i32, f32), lambda: sf.sf_expert_gate_backward(None, x, 0, i32, f32, x),
                 lambda: sf.sf_expert_sort(None, i32, 4, 1, i32, i32, i32, i32), lambda: sf.sf_expert_gather(None, x, i32, i32, i32, x),
                 lambda: sf.sf_expert_gather_backward(None, x, i32, x), lambda: sf.sf_expert_combine(None, x, i32, None, x),
                 lambda: sf.sf_expert_combine_backward(None, x, x, i32, None, i32, i32, x, None)):
        with pytest.raises(sf.SfError) as e:
            call()
        assert e.value.status == sf.SF_ERR_ARG


def test_no_context_is_refused(sf):
    """The C entries look at the context and the sizes before they touch the device."""
    L = sf._lib()
    assert L.sf_mx4_quantise(None, 16, 0, 1, 32, 32, None, None, 1, 16, 16, None) == sf.SF_ERR_ARG
    assert L.sf_mx4_unpack(None, 16, 16, None, 1, 32, 0, 16, 32, None) == sf.SF_ERR_ARG
    assert L.sf_mx4_matmul(None, 16, 16, None, 1, 16, 16, 1, 32, None, 0, 0, 16, 1, None, None) == sf.SF_ERR_ARG
    assert L.sf_mx4_matmul_experts(None, 16, 16, 16, 1, 1, 16, 16, 1, 32, None, 0, 0, 16, 1, None, None) == sf.SF_ERR_ARG
    assert L.sf_expert_gate(None, 16, 0, None, 1, 4, 4, 1, 0, 16, 16, None) == sf.SF_ERR_ARG
    assert L.sf_expert_gate_backward(None, 16, 0, None, 1, 4, 4, 1, 0, 16, 16, 16, 4, None) == sf.SF_ERR_ARG
    assert L.sf_expert_sort(None, 16, None, 1, 1, 1, 1, 1, 16, 16, 16, 16, None, 0, None) == sf.SF_ERR_ARG
    assert L.sf_expert_gather(None, 16, 0, None, 1, 4, 4, 1, 16, 1, 16, 16, 1, 16, 4, None) == sf.SF_ERR_ARG
    assert L.sf_expert_gather_backward(None, 16, 0, 1, 4, 4, 16, None, 1, 1, 16, 4, None) == sf.SF_ERR_ARG
    assert L.sf_expert_combine(None, 16, 0, 1, 4, 4, 16, None, None, 1, 1, 16, 4, None) == sf.SF_ERR_ARG
    assert L.sf_expert_combine_backward(None, 16, 0, 4, 16, 1, 4, 4, 16, None, None, 1, 1, 1, 16, 16, 16, 4, None, None) == sf.SF_ERR_ARG
