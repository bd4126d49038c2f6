"""CPU: refusals of daf_add_rmsnorm and daf_linear_mx, which come before anything touches the GPU."""
import pytest

import paper_2607_21599_amd as daf

FAKE = 0x10000  # an aligned non-null address; never dereferenced on these paths
INVALID, ALIGN, UNSUPPORTED, WORKSPACE = (daf.DAF_ERR_INVALID_ARG, daf.DAF_ERR_ALIGNMENT, daf.DAF_ERR_UNSUPPORTED,
                                          daf.DAF_ERR_WORKSPACE)


def _status(fn, *args):
    with pytest.raises(daf.DafError) as e:
        fn(*args)
    assert daf.daf_last_error()
    return e.value.status


NORM = dict(dtype=daf.DAF_BF16, rows=3, width=64, x=FAKE, delta=2 * FAKE, w=3 * FAKE, eps=1e-6, sum=4 * FAKE,
            y=5 * FAKE, codes=6 * FAKE, scales=7 * FAKE, stream=0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(width=0), UNSUPPORTED), (dict(width=60), UNSUPPORTED),
    (dict(width=40), UNSUPPORTED),  # codes need whole blocks of 32
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(scales=None), INVALID), (dict(codes=None), INVALID),
    (dict(y=None, codes=None, scales=None), INVALID), (dict(delta=None), INVALID), (dict(y=4 * FAKE), INVALID),
    (dict(x=FAKE + 8), ALIGN), (dict(delta=FAKE + 8), ALIGN), (dict(w=FAKE + 8), ALIGN), (dict(sum=FAKE + 8), ALIGN),
    (dict(y=FAKE + 8), ALIGN), (dict(codes=FAKE + 8), ALIGN), (dict(rows=1 << 40), UNSUPPORTED)])
def test_bad_norms(change, status):
    assert _status(daf.daf_add_rmsnorm, *dict(NORM, **change).values()) == status


def test_no_rows_are_no_work():
    daf.daf_add_rmsnorm(*dict(NORM, rows=0, x=None).values())
    daf.daf_linear_mx(0, 64, 64, None, None, None, None, None, None, None, None, 0, 0)
    assert daf.daf_linear_mx_workspace_size(0, 64, 64) == 0


LINEAR = dict(m=3, n=64, k=64, a=FAKE, a_scales=FAKE + 1, w=FAKE, w_scales=FAKE + 3, bias=FAKE, residual=FAKE, c=FAKE,
              ws=FAKE, ws_bytes=1 << 40, stream=0)


@pytest.mark.parametrize("change,status", [
    (dict(m=-1), INVALID), (dict(n=0), INVALID), (dict(n=-5), INVALID), (dict(k=0), UNSUPPORTED),
    (dict(k=48), UNSUPPORTED), (dict(a=None), INVALID), (dict(w=None), INVALID), (dict(w_scales=None), INVALID),
    (dict(c=None), INVALID), (dict(a=FAKE + 8), ALIGN), (dict(w=FAKE + 8), ALIGN), (dict(bias=FAKE + 8), ALIGN),
    (dict(residual=FAKE + 8), ALIGN), (dict(c=FAKE + 8), ALIGN), (dict(m=1 << 40), UNSUPPORTED),
    (dict(m=1 << 20, n=1 << 20), UNSUPPORTED)])
def test_bad_linears(change, status):
    assert _status(daf.daf_linear_mx, *dict(LINEAR, **change).values()) == status


def test_linear_workspace():
    m, n, k = 12, 96, 18944  # few outputs of long sums: K is split
    need = daf.daf_linear_mx_workspace_size(m, n, k)
    assert need > 0 and need % (m * n * 4) == 0
    args = dict(LINEAR, m=m, n=n, k=k)
    assert _status(daf.daf_linear_mx, *dict(args, ws=None).values()) == WORKSPACE
    assert _status(daf.daf_linear_mx, *dict(args, ws_bytes=need - 1).values()) == WORKSPACE
    assert _status(daf.daf_linear_mx, *dict(args, ws=FAKE + 4).values()) == ALIGN
    for bad in ((-1, n, k), (m, 0, k), (m, n, 33)):
        assert daf.daf_linear_mx_workspace_size(*bad) == 0
