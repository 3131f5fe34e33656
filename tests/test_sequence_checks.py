"""What the calls on sequences and on logits refuse, without a device: the binding's looks at its tensors on stand-ins, the library's at its
arguments (refused before anything is launched: the context that it is given is never looked into)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2402_03694_b200 import binding as sf  # noqa: E402
from test_binding_checks import OnDevice, Recorder  # noqa: E402

R, D, N, W, S, V, K = 6, 8, 4, 3, 2, 10, 2


def f32(*s):
    return torch.zeros(*s)


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


@pytest.fixture
def stub(monkeypatch):
    lib, ctx = Recorder(), ctypes.c_void_p(4096)
    monkeypatch.setattr(sf, "_lib", lambda: lib)
    monkeypatch.setitem(sf._ctx_device, ctx.value, 0)
    return lib, ctx


def sequences(device=0):
    return sf.make_sequences(OnDevice(i32(S + 1), device), 5, counts=OnDevice(i32(S), device), slots=OnDevice(i32(S), device))


def calls():
    """name -> (call by named tensors, those tensors)."""
    rows = {"u": f32(R, D), "delta": f32(R, D), "A": f32(D, N), "B": f32(R, N), "C": f32(R, N), "skip": f32(D), "bias": f32(D), "z": f32(R, D)}
    starts = f32((R // 8 + S) * D * N)
    return {
        "conv": (lambda c, q, x, w, y, b, si, so: sf.sf_seq_conv(c, q, x, w, y, bias=b, act=1, state_in=si, state_out=so, stream=7),
                 {"x": f32(R, D), "w": f32(D, W), "y": f32(R, D), "b": f32(D), "si": f32(S, W - 1, D), "so": f32(S, W - 1, D)}),
        "conv backward": (lambda c, q, x, w, dy, work, b, si, ds, dx, dw, db, di: sf.sf_seq_conv_backward(
            c, q, x, w, dy, work, bias=b, state_in=si, d_state=ds, dx_out=dx, dw_out=dw, dbias_out=db, d_state_in_out=di, stream=7),
            {"x": f32(R, D), "w": f32(D, W), "dy": f32(R, D), "work": f32(64), "b": f32(D), "si": f32(S, W - 1, D), "ds": f32(S, W - 1, D), "dx": f32(R, D), "dw": f32(D, W),
             "db": f32(D), "di": f32(S, W - 1, D)}),
        "scan": (lambda c, q, u, delta, A, B, C, skip, bias, z, y, si, so, starts, work: sf.sf_seq_scan(
            c, q, u, delta, A, B, C, y, D=skip, delta_bias=bias, z=z, state_in=si, state_out=so, starts_out=starts, workspace=work, stream=7),
            {**rows, "y": f32(R, D), "si": f32(S, D, N), "so": f32(S, D, N), "starts": starts, "work": f32(64)}),
        "scan backward": (lambda c, q, u, delta, A, B, C, skip, bias, z, dy, starts, work, ds, di, **g: sf.sf_seq_scan_backward(
            c, q, u, delta, A, B, C, dy, starts, work, D=skip, delta_bias=bias, z=z, d_state=ds, d_state_in_out=di, stream=7, **g),
            {**rows, "dy": f32(R, D), "starts": starts, "work": f32(64), "ds": f32(S, D, N), "di": f32(S, D, N), "du_out": f32(R, D), "d_delta_out": f32(R, D),
             "dA_out": f32(D, N), "dB_out": f32(R, N), "dC_out": f32(R, N), "dD_out": f32(D), "d_delta_bias_out": f32(D), "dz_out": f32(R, D)}),
        "logprobs": (lambda c, q, x, labels, lp, h, lse, ids, top, n: sf.sf_label_logprobs(c, x, labels, lp, entropy_out=h, lse_out=lse, top_ids_out=ids, top_logprobs_out=top, n_dev=n, stream=7),
                     {"x": f32(R, V), "labels": i32(R), "lp": f32(R), "h": f32(R), "lse": f32(R), "ids": i32(R, K), "top": f32(R, K), "n": i32(1)}),
        "logprobs backward": (lambda c, q, x, labels, lse, d, dl, h, dh, ids, dt, n: sf.sf_label_logprobs_backward(
            c, x, labels, lse, d, d_logprob=dl, entropy=h, d_entropy=dh, top_ids=ids, d_top_logprobs=dt, n_dev=n, stream=7),
            {"x": f32(R, V), "labels": i32(R), "lse": f32(R), "d": f32(R, V), "dl": f32(R), "h": f32(R), "dh": f32(R), "ids": i32(R, K), "dt": f32(R, K), "n": i32(1)}),
    }


@pytest.mark.parametrize("name", list(calls()))
def test_every_tensor_has_to_be_on_the_contexts_device_and_of_its_shape_and_type(stub, name):
    lib, ctx = stub
    call, tensors = calls()[name]
    q = sequences()
    call(ctx, q, **{k: OnDevice(t) for k, t in tensors.items()})
    assert len(lib.calls) == 1

    def refused(k, t, device=0):
        with pytest.raises(sf.SfError) as e:
            call(ctx, q, **{o: OnDevice(t if o == k else v, device if o == k else 0) for o, v in tensors.items()})
        assert e.value.status == sf.SF_ERR_ARG, (k, tuple(t.shape))
    for k, t in tensors.items():
        refused(k, t, 1)                                   # another device
        refused(k, t, -1)                                  # host memory
        if k in ("work", "n"):
            continue
        refused(k, t.double() if t.is_floating_point() else t.long())
        if k == "starts":
            refused(k, t[:-1])
        elif k in ("u", "x"):                              # what the sizes are taken from: the others no longer fit
            refused(k, f32(t.shape[0] + 1, t.shape[1]))
            refused(k, torch.zeros(t.shape[1], t.shape[0]).t())
        else:
            refused(k, torch.zeros(t.shape[0] + 1, *t.shape[1:], dtype=t.dtype))
            if t.dim() == 2:
                refused(k, torch.zeros(t.shape[1], t.shape[0], dtype=t.dtype).t())
    assert len(lib.calls) == 1


@pytest.mark.parametrize("name", ["conv", "conv backward", "scan", "scan backward"])
def test_sequences_of_another_device(stub, name):
    lib, ctx = stub
    call, tensors = calls()[name]
    with pytest.raises(sf.SfError):
        call(ctx, sequences(1), **{k: OnDevice(t) for k, t in tensors.items()})
    assert not lib.calls


def test_sequences_are_looked_at(stub):
    for bad in (lambda: sf.make_sequences(i32(3), 5), lambda: sf.make_sequences(OnDevice(i32(0)), 5), lambda: sf.make_sequences(OnDevice(i32(3)), 0),
                lambda: sf.make_sequences(OnDevice(f32(3)), 5), lambda: sf.make_sequences(OnDevice(i32(3)), 5, counts=OnDevice(i32(1))),
                lambda: sf.make_sequences(OnDevice(i32(3)), 5, slots=OnDevice(i32(1))), lambda: sf.make_sequences(OnDevice(i32(3)), 5, counts=OnDevice(i32(2), 1)),
                lambda: sf.make_sequences(OnDevice(i32(3)), 2 ** 32)):
        with pytest.raises(sf.SfError):
            bad()


# ---- the library itself ------------------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    from paper_2402_03694_b200 import build
    build.build()
    return sf._lib()


P = 1 << 20                                                # an address on every boundary; nothing follows it


def seq(n_seq=2, max_len=5, offsets=P, counts=None, slots=None):
    return sf.sf_sequences(offsets, counts, slots, n_seq, max_len)


def test_convolution_refusals(lib):
    good = dict(ctx=P, seq=seq(), x=P, dtype=0, rows=6, D=8, ldx=8, w=P, bias=P, W=4, act=1, state_in=P, state_out=P, n_slots=2, y=P, ldy=8, stream=0)
    bad = [dict(ctx=None), dict(seq=None), dict(x=None), dict(w=None), dict(y=None), dict(dtype=3), dict(dtype=-1), dict(D=0), dict(D=2 ** 24 + 1), dict(ldx=7), dict(ldy=7), dict(W=0),
           dict(W=9), dict(act=2), dict(rows=sf.SF_SEQ_MAX_ROWS + 1), dict(n_slots=2 ** 31), dict(x=P + 2), dict(w=P + 1), dict(bias=P + 2), dict(state_in=P + 1), dict(y=P + 1), dict(dtype=1, x=P + 1),
           dict(seq=seq(max_len=0)), dict(seq=seq(max_len=sf.SF_SEQ_MAX_ROWS + 1)), dict(seq=seq(offsets=None)), dict(seq=seq(offsets=P + 2)), dict(seq=seq(counts=P + 1)), dict(seq=seq(slots=P + 1)), dict(seq=seq(n_seq=2 ** 31))]
    for b in bad:
        assert lib.sf_seq_conv(*{**good, **b}.values()) == sf.SF_ERR_ARG, b
    back = dict(ctx=P, seq=seq(), x=P, dtype=0, rows=6, D=8, ldx=8, w=P, bias=P, W=4, act=1, state_in=P, dy=P, lddy=8, d_state=P, n_slots=2, dx=P, lddx=8, dw=P, db=P, di=P, work=P,
                bytes=0, stream=0)
    for b in [b for b in bad if not {"y", "ldy"} & set(b)] + [dict(dy=None), dict(lddy=7), dict(lddx=7), dict(dx=None, dw=None, db=None, di=None), dict(work=P + 1), dict(dw=P + 2)]:
        assert lib.sf_seq_conv_backward(*{**back, **b}.values()) == sf.SF_ERR_ARG, b


def test_scan_refusals(lib):
    def rows(**kw):
        v = dict(u=P, delta=P, B=P, C=P, z=P, ldu=8, ld_delta=8, ldb=8, ldc=8, ldz=8, A=P, D_skip=P, delta_bias=P, D=8, N=4, G=2, dtype=0, softplus=1)
        return sf.sf_scan_rows(*{**v, **kw}.values())
    good = dict(ctx=P, seq=seq(), rows_in=rows(), rows=6, si=P, so=P, n_slots=2, starts=P, y=P, ldy=8, work=None, bytes=0, stream=0)
    inside = [dict(u=None), dict(delta=None), dict(B=None), dict(C=None), dict(A=None), dict(ldu=7), dict(ld_delta=7), dict(ldz=7), dict(ldb=7), dict(ldc=7), dict(D=0), dict(N=0),
              dict(N=65), dict(G=0), dict(G=3), dict(D=2 ** 24 + 2), dict(dtype=3), dict(u=P + 1), dict(A=P + 2), dict(D_skip=P + 1), dict(z=P + 2), dict(B=P + 2)]
    bad = [dict(rows_in=rows(**kw)) for kw in inside] + [dict(ctx=None), dict(seq=None), dict(rows_in=None), dict(rows=2 ** 31), dict(seq=seq(max_len=0)), dict(seq=seq(offsets=P + 1))]
    for b in bad + [dict(y=None), dict(ldy=7), dict(y=P + 1), dict(si=P + 1), dict(starts=P + 2), dict(n_slots=2 ** 31), dict(seq=seq(n_seq=1, max_len=10000))]:      # (the last: in parts, no workspace)
        assert lib.sf_seq_scan(*{**good, **b}.values()) == sf.SF_ERR_ARG, b

    def grads(**kw):
        v = dict(du=P, d_delta=P, dB=P, dC=P, dz=P, lddu=8, ldd_delta=8, lddb=8, lddc=8, lddz=8, dA=P, dD=P, db=P)
        return sf.sf_scan_grads(*{**v, **kw}.values())
    back = dict(ctx=P, seq=seq(), rows_in=rows(), rows=6, dy=P, lddy=8, starts=P, ds=P, di=P, n_slots=2, out=grads(), work=P, bytes=0, stream=0)
    more = [dict(out=grads(**kw)) for kw in (dict(lddu=7), dict(ldd_delta=7), dict(lddb=7), dict(lddc=7), dict(lddz=7), dict(du=P + 1), dict(dA=P + 2), dict(dB=P + 1))]
    for b in bad + more + [dict(dy=None), dict(starts=None), dict(out=None), dict(lddy=7), dict(work=None), dict(work=P + 1), dict(rows_in=rows(z=None)), dict()]:          # (the last: workspace too small)
        assert lib.sf_seq_scan_backward(*{**back, **b}.values()) == sf.SF_ERR_ARG, b


def test_logprob_refusals(lib):
    good = dict(ctx=P, x=P, dtype=0, n_dev=None, n=6, V=10, ld=10, scale=1.0, labels=P, lp=P, h=P, lse=P, k=2, ids=P, top=P, stream=0)
    bad = [dict(ctx=None), dict(x=None), dict(dtype=3), dict(V=0), dict(V=0x7FF00001, ld=2 ** 31), dict(ld=9), dict(n=2 ** 31), dict(k=33, V=100, ld=100), dict(k=11), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=2e30),
           dict(scale=float("nan")), dict(x=P + 2), dict(labels=P + 1), dict(n_dev=P + 1)]
    for b in bad + [dict(labels=None), dict(lp=None, h=None, lse=None, ids=None, top=None), dict(lp=None, h=None, lse=None, k=0), dict(lp=P + 1), dict(ids=None, top=None), dict(top=P + 2)]:
        assert lib.sf_label_logprobs(*{**good, **b}.values()) == sf.SF_ERR_ARG, b
    back = dict(ctx=P, x=P, dtype=0, n_dev=None, n=6, V=10, ld=10, scale=1.0, labels=P, lse=P, dl=P, h=P, dh=P, k=2, ids=P, dt=P, d=P, ldd=10, stream=0)
    for b in bad + [dict(labels=None), dict(lse=None), dict(d=None), dict(ldd=9), dict(h=None), dict(ids=None), dict(dl=P + 1), dict(d=P + 2)]:
        assert lib.sf_label_logprobs_backward(*{**back, **b}.values()) == sf.SF_ERR_ARG, b


def test_nothing_to_do_is_no_error(lib):
    assert lib.sf_label_logprobs(P, None, 0, None, 0, 10, 10, 1.0, P, P, P, P, 2, P, P, 0) == sf.SF_OK
    assert lib.sf_label_logprobs_backward(P, None, 0, None, 0, 10, 10, 1.0, None, None, None, None, None, 0, None, None, None, 10, 0) == sf.SF_OK
    assert lib.sf_seq_conv(P, seq(n_seq=0, offsets=None), None, 0, 0, 8, 8, P, None, 4, 0, None, None, 0, None, 8, 0) == sf.SF_OK


def test_sizes_of_workspaces(lib):
    z = ctypes.c_size_t()
    assert lib.sf_seq_scan_workspace(64, 128, 8192, 1024, 16, 1, 0, ctypes.byref(z)) == sf.SF_OK and z.value == 0       # many sequences: in one go
    assert lib.sf_seq_scan_workspace(1, 8192, 8192, 1024, 16, 1, 0, ctypes.byref(z)) == sf.SF_OK and z.value > 0
    assert lib.sf_seq_scan_starts(3, 100, 8, 4, ctypes.byref(z)) == sf.SF_OK and z.value == (100 // 8 + 3) * 32
    for bad in ((1, 0, 8, 8, 4, 1), (1, 4, 8, 0, 4, 1), (1, 4, 8, 8, 65, 1), (1, 4, 8, 8, 4, 3), (2 ** 31, 4, 8, 8, 4, 1), (1, 4, 2 ** 31, 8, 4, 1)):
        assert lib.sf_seq_scan_workspace(*bad, 0, ctypes.byref(z)) == sf.SF_ERR_ARG, bad
    assert lib.sf_seq_scan_workspace(1, 4, 8, 8, 4, 1, 0, None) == sf.SF_ERR_ARG
    assert lib.sf_seq_conv_backward_workspace(1, 4, 8, 9, ctypes.byref(z)) == sf.SF_ERR_ARG
    for n, L, d, w in ((1, 1, 1, 1), (1000, 128, 256, 4), (1, 100000, 7, 8)):
        assert sf.sf_seq_conv_backward_workspace(n, L, d, w) >= d * (w + 1) * 4
    with pytest.raises(sf.SfError):
        sf.sf_seq_scan_workspace(1, 4, 8, 8, 4, -1)
    with pytest.raises(sf.SfError):
        sf.sf_seq_scan_starts(1, 2 ** 33, 8, 4)
