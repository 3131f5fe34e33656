"""What the packed-row and expert calls look at before they reach the library, on stand-in tensors: no device needed, nothing launched."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2402_03694_b200 import binding as sf  # noqa: E402


class OnDevice:
    """A host tensor that says it lives on a device."""

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def get_device(self):
        return self.device_index

    @property
    def is_cuda(self):
        return self.device_index >= 0

    def __getattr__(self, name):
        return getattr(self.t, name)


class Recorder:
    """Stands for the library: every call succeeds and is counted."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name in ("sf_strerror", "sf_last_cuda_error"):
                return b"refused"
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def stub(monkeypatch):
    lib, ctx = Recorder(), ctypes.c_void_p(4096)
    monkeypatch.setattr(sf, "_lib", lambda: lib)
    monkeypatch.setitem(sf._ctx_device, ctx.value, 0)
    return lib, ctx


N, K, E, D, CAP = 6, 64, 4, 8, 40


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def f32(*s):
    return torch.zeros(*s)


def u8(*s):
    return torch.zeros(*s, dtype=torch.uint8)


def packed(rows, k, experts=1):
    d, s = sf._mx4_bytes(rows, k)
    return u8(experts * rows * d), u8(experts * s)


def calls():
    """name -> (call by named tensors, those tensors)."""
    a, sa = packed(N, K)
    w, sw = packed(D, K)
    we, swe = packed(D, K, E)
    o, so = packed(N, D)
    pairs = {"ids": i32(N, 2), "weights": f32(N, 2)}
    plan = {"row_of_pair": i32(N, 2), "offsets": i32(E + 1), "counts": i32(E)}
    return {
        "quantise": (lambda c, x, data, scales, row_ids, n: sf.sf_mx4_quantise(c, x, data, scales, row_ids=row_ids, n_rows_dev=n, stream=7),
                     {"x": f32(N, K), "data": a, "scales": sa, "row_ids": i32(N), "n": i32(1)}),
        "unpack": (lambda c, x, data, scales, n: sf.sf_mx4_unpack(c, data, scales, x, n_rows_dev=n, stream=7),
                   {"x": f32(N, K), "data": a, "scales": sa, "n": i32(1)}),
        "matmul": (lambda c, a, sa, w, sw, out, bias, n: sf.sf_mx4_matmul(c, a, sa, w, sw, K, out, bias=bias, n_rows_dev=n, stream=7),
                   {"a": a, "sa": sa, "w": w, "sw": sw, "out": f32(N, D), "bias": f32(D), "n": i32(1)}),
        "matmul packed again": (lambda c, a, sa, w, sw, out, so: sf.sf_mx4_matmul(c, a, sa, w, sw, K, out, out_scales=so, N=D, stream=7),
                                {"a": a, "sa": sa, "w": w, "sw": sw, "out": o.view(N, -1), "so": so}),
        "matmul by expert": (lambda c, a, sa, w, sw, out, bias, offsets: sf.sf_mx4_matmul_experts(c, a, sa, w, sw, K, offsets, out, bias=bias, stream=7),
                             {"a": a, "sa": sa, "w": we, "sw": swe, "out": f32(N, D), "bias": f32(E, D), "offsets": i32(E + 1)}),
        "matmul by expert packed again": (lambda c, a, sa, w, sw, out, so, offsets: sf.sf_mx4_matmul_experts(c, a, sa, w, sw, K, offsets, out, out_scales=so, N=D, stream=7),
                                          {"a": a, "sa": sa, "w": we, "sw": swe, "out": o.view(N, -1), "so": so, "offsets": i32(E + 1)}),
        "gate": (lambda c, scores, ids, weights, n: sf.sf_expert_gate(c, scores, 0, ids, weights, n_dev=n, stream=7),
                 {"scores": f32(N, E), "n": i32(1), **pairs}),
        "gate backward": (lambda c, scores, ids, weights, d, n: sf.sf_expert_gate_backward(c, scores, 0, ids, weights, d, n_dev=n, stream=7),
                          {"scores": f32(N, E), "d": f32(N, E), "n": i32(1), **pairs}),
        "sort": (lambda c, ids, offsets, counts, flow, row_of_pair, work, n: sf.sf_expert_sort(c, ids, E, 1, offsets, counts, flow, row_of_pair, work, n_dev=n, stream=7),
                 {"ids": i32(N, 2), "flow": i32(CAP), "work": u8(64), "n": i32(1), **plan}),
        "gather": (lambda c, x, row_of_pair, offsets, counts, rows, n: sf.sf_expert_gather(c, x, row_of_pair, offsets, counts, rows, n_dev=n, stream=7),
                   {"x": f32(N, D), "rows": f32(CAP, D), "n": i32(1), **plan}),
        "gather backward": (lambda c, rows, row_of_pair, dx, n: sf.sf_expert_gather_backward(c, rows, row_of_pair, dx, n_dev=n, stream=7),
                            {"rows": f32(CAP, D), "row_of_pair": i32(N, 2), "dx": f32(N, D), "n": i32(1)}),
        "combine": (lambda c, rows, row_of_pair, weights, y, n: sf.sf_expert_combine(c, rows, row_of_pair, weights, y, n_dev=n, stream=7),
                    {"rows": f32(CAP, D), "row_of_pair": i32(N, 2), "weights": f32(N, 2), "y": f32(N, D), "n": i32(1)}),
        "combine backward": (lambda c, dy, rows, row_of_pair, weights, offsets, counts, d_rows, d_w, n:
                             sf.sf_expert_combine_backward(c, dy, rows, row_of_pair, weights, offsets, counts, d_rows, d_w, n_dev=n, stream=7),
                             {"dy": f32(N, D), "rows": f32(CAP, D), "weights": f32(N, 2), "d_rows": f32(CAP, D), "d_w": f32(N, 2), "n": i32(1), **plan}),
    }


@pytest.mark.parametrize("name", list(calls()))
def test_every_tensor_has_to_be_on_the_contexts_device(stub, name):
    lib, ctx = stub
    call, tensors = calls()[name]
    call(ctx, **{k: OnDevice(t) for k, t in tensors.items()})
    assert len(lib.calls) == 1
    for k in tensors:
        for device in (1, -1):                           # another device, host memory
            with pytest.raises(sf.SfError) as e:
                call(ctx, **{q: OnDevice(t, device if q == k else 0) for q, t in tensors.items()})
            assert e.value.status == sf.SF_ERR_ARG, k
    with pytest.raises(sf.SfError):                      # a whole call on another device
        call(ctx, **{q: OnDevice(t, 1) for q, t in tensors.items()})
    for other in (None, ctypes.c_void_p(8192)):          # no context, one that is not there (any more)
        with pytest.raises(sf.SfError):
            call(other, **{q: OnDevice(t) for q, t in tensors.items()})
    assert len(lib.calls) == 1


BIG = (1 << 32) + 3                                      # its low half would be a size of 3


def meta(*s, t=torch.float32):
    """A tensor of any size without memory."""
    return OnDevice(torch.empty(*s, dtype=t, device="meta"))


@pytest.mark.parametrize("call", [
    lambda c: sf.sf_mx4_quantise(c, meta(BIG, 1), meta(BIG * 16, t=torch.uint8), meta(BIG * 8, t=torch.uint8), stream=7),
    lambda c: sf.sf_mx4_quantise(c, meta(1, BIG), meta(BIG, t=torch.uint8), meta(BIG * 8, t=torch.uint8), stream=7),
    lambda c: sf.sf_mx4_quantise(c, meta(9, 1), meta(BIG * 16, t=torch.uint8), meta(BIG * 8, t=torch.uint8), row_ids=meta(BIG, t=torch.int32), stream=7),
    lambda c: sf.sf_mx4_unpack(c, meta(BIG * 16, t=torch.uint8), meta(BIG * 8, t=torch.uint8), meta(BIG, 1), stream=7),
    lambda c: sf.sf_mx4_matmul(c, meta(BIG * 16, t=torch.uint8), meta(BIG * 8, t=torch.uint8), meta(64, t=torch.uint8), meta(512, t=torch.uint8), 32, meta(BIG, 4), stream=7),
    lambda c: sf.sf_mx4_matmul(c, meta(BIG * 2, t=torch.uint8), meta(BIG * 8, t=torch.uint8), meta(BIG * 4, t=torch.uint8), meta(BIG * 8, t=torch.uint8), BIG, meta(1, 4), stream=7),
    lambda c: sf.sf_mx4_matmul(c, meta(BIG * 16, t=torch.uint8), meta(BIG * 8, t=torch.uint8), meta(64, t=torch.uint8), meta(512, t=torch.uint8), 32, meta(BIG, 16, t=torch.uint8),
                               out_scales=meta(BIG * 8, t=torch.uint8), N=4, stream=7),
    lambda c: sf.sf_mx4_matmul_experts(c, meta(64, t=torch.uint8), meta(512, t=torch.uint8), meta(BIG * 64, t=torch.uint8), meta(BIG * 512, t=torch.uint8), 32, meta(BIG + 1, t=torch.int32),
                                       meta(4, 4), stream=7),
    lambda c: sf.sf_expert_gate(c, meta(BIG, 4), 0, meta(BIG, 1, t=torch.int32), meta(BIG, 1), stream=7),
    lambda c: sf.sf_expert_gate(c, meta(1, 4), 0, meta(1, BIG, t=torch.int32), meta(1, BIG), stream=7),
    lambda c: sf.sf_expert_gate_backward(c, meta(BIG, 4), 0, meta(BIG, 1, t=torch.int32), meta(BIG, 1), meta(BIG, 4), stream=7),
    lambda c: sf.sf_expert_gate_backward(c, meta(1, 4), 0, meta(1, BIG, t=torch.int32), meta(1, BIG), meta(1, 4), stream=7),
    lambda c: sf.sf_expert_sort(c, meta(BIG, 1, t=torch.int32), 4, 1, meta(5, t=torch.int32), meta(4, t=torch.int32), meta(9, t=torch.int32), meta(BIG, 1, t=torch.int32), stream=7),
    lambda c: sf.sf_expert_sort(c, meta(3, 1, t=torch.int32), 4, 1, meta(5, t=torch.int32), meta(4, t=torch.int32), meta(BIG, t=torch.int32), meta(3, 1, t=torch.int32), stream=7),
    lambda c: sf.sf_expert_sort(c, meta(3, 1, t=torch.int32), 4, (1 << 32) + 128, meta(5, t=torch.int32), meta(4, t=torch.int32), meta(9, t=torch.int32), meta(3, 1, t=torch.int32), stream=7),
    lambda c: sf.sf_expert_gather(c, meta(BIG, 4), meta(BIG, 1, t=torch.int32), meta(5, t=torch.int32), meta(4, t=torch.int32), meta(9, 4), stream=7),
    lambda c: sf.sf_expert_gather(c, meta(3, 4), meta(3, 1, t=torch.int32), meta(5, t=torch.int32), meta(4, t=torch.int32), meta(BIG, 4), stream=7),
    lambda c: sf.sf_expert_gather(c, meta(3, 4), meta(3, 1, t=torch.int32), meta(BIG + 1, t=torch.int32), meta(BIG, t=torch.int32), meta(9, 4), stream=7),
    lambda c: sf.sf_expert_gather_backward(c, meta(9, 4), meta(BIG, 1, t=torch.int32), meta(BIG, 4), stream=7),
    lambda c: sf.sf_expert_combine(c, meta(BIG, 4), meta(3, 1, t=torch.int32), None, meta(3, 4), stream=7),
    lambda c: sf.sf_expert_combine(c, meta(9, 4), meta(3, BIG, t=torch.int32), None, meta(3, 4), stream=7),
    lambda c: sf.sf_expert_combine_backward(c, meta(BIG, 4), meta(9, 4), meta(BIG, 1, t=torch.int32), None, meta(5, t=torch.int32), meta(4, t=torch.int32), None, meta(BIG, 1), stream=7),
    lambda c: sf.sf_expert_combine_backward(c, meta(3, 4), meta(9, 4), meta(3, 1, t=torch.int32), None, meta(BIG + 1, t=torch.int32), meta(BIG, t=torch.int32), None, meta(3, 1), stream=7),
    lambda c: sf.sf_mx4_sizes(BIG, 64),
    lambda c: sf.sf_mx4_sizes(3, BIG),
    lambda c: sf.sf_expert_sort_workspace(BIG, 1, 4),
    lambda c: sf.sf_expert_sort_workspace(3, 1, BIG)])
def test_sizes_past_32_bits_are_refused(stub, call):
    """Their low halves are sizes that the library would take: a part of the rows would be done and the call succeed."""
    lib, ctx = stub
    with pytest.raises(sf.SfError) as e:
        call(ctx)
    assert e.value.status == sf.SF_ERR_ARG and lib.calls == []


def test_weights_gradient_alone_needs_no_segments(stub):
    """Offsets and counts name the rows that only fill a segment of d_rows: without d_rows a call may leave them out."""
    lib, ctx = stub
    dy, rows, at, d_w = (OnDevice(t) for t in (f32(N, D), f32(CAP, D), i32(N, 2), f32(N, 2)))
    sf.sf_expert_combine_backward(ctx, dy, rows, at, None, None, None, None, d_w, stream=7)
    assert lib.calls == ["sf_expert_combine_backward"]
    with pytest.raises((sf.SfError, AttributeError)):
        sf.sf_expert_combine_backward(ctx, dy, rows, at, None, None, None, rows, d_w, stream=7)
    assert len(lib.calls) == 1
