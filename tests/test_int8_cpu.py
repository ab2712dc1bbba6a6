"""st_quantize_rows, st_int8_matmul and st_set_frozen_features_int8 refuse bad arguments on the host, before any launch.  No GPU needed."""
import pytest
import torch

import paper_2003_10735_b200 as st
from paper_2003_10735_b200 import build as st_build


@pytest.fixture(scope="module")
def lib():
    st_build.build()
    return st.load_library()


FAKE = 1 << 20      # never read: every call below is refused before a pointer is looked at


@pytest.mark.parametrize("kw,status", [
    (dict(x_type=3), st.ST_ERR_INVALID_ARG), (dict(x_type=-1), st.ST_ERR_INVALID_ARG), (dict(rows=-1), st.ST_ERR_INVALID_ARG),
    (dict(cols=0), st.ST_ERR_INVALID_ARG), (dict(row_stride=-8), st.ST_ERR_INVALID_ARG), (dict(col_stride=-1), st.ST_ERR_INVALID_ARG),
    (dict(ldq=7), st.ST_ERR_INVALID_ARG), (dict(rows=1 << 31), st.ST_ERR_UNSUPPORTED), (dict(cols=1 << 31, ldq=1 << 31), st.ST_ERR_UNSUPPORTED),
    (dict(rows=1 << 30, row_stride=1 << 60), st.ST_ERR_UNSUPPORTED), (dict(rows=1 << 30, ldq=1 << 60), st.ST_ERR_UNSUPPORTED)])
def test_quantize_refuses(lib, kw, status):
    a = dict(x_type=0, rows=4, cols=8, row_stride=8, col_stride=1, ldq=8)
    a.update(kw)
    got = lib.st_quantize_rows(FAKE, a["x_type"], a["rows"], a["cols"], a["row_stride"], a["col_stride"], FAKE, a["ldq"], FAKE, None)
    assert got == status and "st_quantize_rows" in st.st_last_error(None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), st.ST_ERR_INVALID_ARG), (dict(N=-1), st.ST_ERR_INVALID_ARG), (dict(K=0), st.ST_ERR_INVALID_ARG), (dict(y_type=7), st.ST_ERR_INVALID_ARG),
    (dict(relu=2), st.ST_ERR_INVALID_ARG), (dict(ldx=15), st.ST_ERR_INVALID_ARG), (dict(ldw=15), st.ST_ERR_INVALID_ARG), (dict(ldy=3), st.ST_ERR_INVALID_ARG),
    (dict(K=131072, ldx=131072, ldw=131072), st.ST_ERR_UNSUPPORTED), (dict(M=1 << 31), st.ST_ERR_UNSUPPORTED), (dict(N=1 << 30, ldy=1 << 30), st.ST_ERR_UNSUPPORTED),
    (dict(M=1 << 30, ldx=1 << 50), st.ST_ERR_UNSUPPORTED)])
def test_matmul_refuses(lib, kw, status):
    a = dict(M=4, N=4, K=16, ldx=16, ldw=16, ldy=4, relu=0, y_type=0)
    a.update(kw)
    got = lib.st_int8_matmul(FAKE, a["ldx"], FAKE, FAKE, a["ldw"], FAKE, None, a["relu"], a["M"], a["N"], a["K"], FAKE, a["y_type"], a["ldy"], None)
    assert got == status and "st_int8_matmul" in st.st_last_error(None)


def test_nothing_to_do(lib):
    assert lib.st_quantize_rows(None, 0, 0, 8, 8, 1, None, 8, None, None) == st.ST_OK
    assert lib.st_int8_matmul(None, 16, None, None, 16, None, None, 0, 0, 4, 16, None, 0, 4, None) == st.ST_OK
    assert lib.st_int8_matmul(None, 16, None, None, 16, None, None, 0, 4, 0, 16, None, 0, 4, None) == st.ST_OK
    assert lib.st_set_frozen_features_int8(None, 0, None, 16, None, None, 16, None, None, 0, 16) == st.ST_ERR_INVALID_ARG


def test_binding_checks_types_and_shapes(lib):
    q, s, y = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4), torch.zeros(4, 4)
    with pytest.raises(TypeError):
        st.st_quantize_rows(torch.zeros(4, 16, dtype=torch.float64), q, s)
    with pytest.raises(TypeError):
        st.st_quantize_rows(torch.zeros(64), q, s)
    with pytest.raises(ValueError):
        st.st_quantize_rows(torch.zeros(4, 15), q, s)
    with pytest.raises(ValueError):
        st.st_quantize_rows(torch.zeros(4, 16), q, s[:3])
    with pytest.raises(TypeError):
        st.st_quantize_rows(torch.zeros(4, 16), q.t().contiguous().t(), s)          # columns contiguous instead of rows
    with pytest.raises(ValueError):
        st.st_int8_matmul(q, s, q[:, :8], s, y)
    with pytest.raises(ValueError):
        st.st_int8_matmul(q, s, q, s, y[:3])
    with pytest.raises(TypeError):
        st.st_int8_matmul(q, s, q, s, y.double())
    with pytest.raises(TypeError):
        st.st_int8_matmul(q.float(), s, q, s, y)
    with pytest.raises(ValueError):
        st.st_int8_matmul(q, s, q, s, y, bias=s[:2])
