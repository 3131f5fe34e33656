"""Memory that the calls on sequences are given, without a device: one pool read and written is taken, pools that overlap in part are refused; the binding's sizes are the header's and
the library's."""
import os
import re

import pytest

torch = pytest.importorskip("torch")

from paper_2402_03694_b200 import binding as sf  # noqa: E402

P = 1 << 20                                                # an address on every boundary; nothing follows it


@pytest.fixture(scope="module")
def lib():
    from paper_2402_03694_b200 import build
    build.build()
    return sf._lib()


def seq(n_seq):
    return sf.sf_sequences(P, None, None, n_seq, 5)


def test_pools_that_overlap_in_part_are_refused(lib):
    conv = dict(ctx=P, seq=seq(0), x=P, dtype=sf.SF_BF16, rows=6, D=8, ldx=8, w=P, bias=P, W=4, act=1, state_in=P, state_out=P, n_slots=2, y=P, ldy=8, stream=0)
    one = 3 * 8 * 2                                        # bytes of a state
    call = lambda **kw: lib.sf_seq_conv(*{**conv, **kw}.values())  # noqa: E731
    assert call() == sf.SF_OK                              # (no sequences: what is not refused returns before anything is launched)
    assert call(state_out=P + 2 * one) == sf.SF_OK and call(state_in=P + 2 * one) == sf.SF_OK
    # with sequences the call looks at its pools before it touches a device
    for kw in (dict(state_out=P + one), dict(state_in=P + one), dict(state_out=P + 2 * one - 2)):
        assert call(seq=seq(2), **kw) == sf.SF_ERR_ARG, kw
    back = dict(ctx=P, seq=seq(2), x=P, dtype=sf.SF_BF16, rows=6, D=8, ldx=8, w=P, bias=P, W=4, act=1, state_in=None, dy=P, lddy=8, d_state=P, n_slots=2, dx=P, lddx=8, dw=None, db=None, di=P,
                work=None, bytes=0, stream=0)
    for kw in (dict(di=P + one), dict(d_state=P + one), dict(state_in=P + one, d_state=None)):
        assert lib.sf_seq_conv_backward(*{**back, **kw}.values()) == sf.SF_ERR_ARG, kw
    rows = sf.sf_scan_rows(P, P, P, P, P, 8, 8, 8, 8, 8, P, P, P, 8, 4, 2, 0, 1)
    scan = dict(ctx=P, seq=seq(2), rows_in=rows, rows=6, si=P, so=P, n_slots=2, starts=P, y=P, ldy=8, work=None, bytes=0, stream=0)
    for kw in (dict(so=P + 128), dict(si=P + 128), dict(so=P + 252)):
        assert lib.sf_seq_scan(*{**scan, **kw}.values()) == sf.SF_ERR_ARG, kw
    assert lib.sf_seq_scan(*{**scan, "seq": seq(0), "so": P + 256}.values()) == sf.SF_OK
    grads = sf.sf_scan_grads(P, P, P, P, P, 8, 8, 8, 8, 8, P, P, P)
    need = sf.sf_seq_scan_workspace(2, 5, 6, 8, 4, 2, backward=True)
    back = dict(ctx=P, seq=seq(2), rows_in=rows, rows=6, dy=P, lddy=8, starts=P, ds=P, di=P, n_slots=2, out=grads, work=P, bytes=need, stream=0)
    for kw in (dict(di=P + 128), dict(ds=P + 128)):
        assert lib.sf_seq_scan_backward(*{**back, **kw}.values()) == sf.SF_ERR_ARG, kw


def test_the_bindings_constants_are_the_headers(lib):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "serveflow.h")).read()
    defined = dict(re.findall(r"#define\s+(SF_\w+)\s+(-?\d+)u?\s", text))
    for name in ("SF_ACT_NONE", "SF_ACT_SILU", "SF_SEQ_MAX_ROWS", "SF_SCAN_MAX_STATES", "SF_SCAN_EVERY", "SF_MAX_TOP"):
        assert int(defined[name]) == getattr(sf, name), name


class Tensor:
    """As much of a device tensor as the check of the kept states looks at."""
    dtype = torch.float32

    def __init__(self, n):
        self.n = n

    def get_device(self):
        return 0

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P


@pytest.mark.parametrize("n_seq,rows,D,N", [(1, 0, 3, 1), (2, 7, 8, 4), (5, 8, 1, 16), (3, 100, 8, 64), (9, 12345, 77, 5)])
def test_room_for_kept_states_is_what_the_library_asks_for(lib, n_seq, rows, D, N):
    need = sf.sf_seq_scan_starts(n_seq, rows, D, N)
    sf._types()
    assert sf._starts(Tensor(need), rows, n_seq, D, N, 0, "scan") == P
    with pytest.raises(sf.SfError):
        sf._starts(Tensor(need - 1), rows, n_seq, D, N, 0, "scan")
