"""st_adamw_create and its companions refuse bad descriptions on the host, before any CUDA call.  No GPU needed."""
import ctypes

import pytest
import torch

import paper_2003_10735_b200 as st
from paper_2003_10735_b200 import build as st_build


@pytest.fixture(scope="module")
def lib():
    st_build.build()
    return st.load_library()


def _create(lib, tensors=None, **kw):
    d = dict(n_tensors=1, state_bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=0.0, skip_nonfinite=0, first_step=0)
    d.update(kw)
    desc = st.st_adamw_desc(*[d[f] for f, _ in st.st_adamw_desc._fields_[:-1]], None)
    out = ctypes.c_void_p(1)
    table = tensors if tensors is not None else (st.st_adamw_tensor * 1)()
    status = lib.st_adamw_create(ctypes.byref(desc), table, ctypes.byref(out))
    return status, out.value


@pytest.mark.parametrize("kw", [
    dict(n_tensors=0), dict(n_tensors=-1), dict(n_tensors=65536), dict(state_bits=16), dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")),
    dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=1e-40), dict(eps=float("nan")),
    dict(eps=1e39), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(max_norm=float("inf")), dict(skip_nonfinite=2), dict(first_step=-1)])
def test_create_refuses_descriptions(lib, kw):
    status, handle = _create(lib, **kw)
    assert status == st.ST_ERR_INVALID_ARG and handle is None
    assert "st_adamw_create" in st.st_adamw_last_error(None) and st.st_adamw_last_error(None) == st.st_last_error(None)


@pytest.mark.parametrize("eps,refused", [(2.0 ** 100, False), (2.0 ** 101, True), (5e37, True), (3.4e38, True)])
def test_an_eps_that_leaves_no_room_for_the_root_is_refused(lib, eps, refused):
    """Denominators above 2^125 are those of roots that have left fp32; an eps of that size would be taken for one."""
    empty = (st.st_adamw_tensor * 1)(st.st_adamw_tensor(param_type=7))         # refused for its type where eps is not
    status, handle = _create(lib, empty, eps=eps)
    assert status != st.ST_OK and handle is None
    assert ("needs lr" in st.st_adamw_last_error(None)) == refused


def test_null_arguments(lib):
    out = ctypes.c_void_p()
    assert lib.st_adamw_create(None, None, ctypes.byref(out)) == st.ST_ERR_INVALID_ARG
    assert lib.st_adamw_step(None, 1.0, None) == st.ST_ERR_INVALID_ARG
    assert lib.st_adamw_set_grads(None, None) == st.ST_ERR_INVALID_ARG
    assert lib.st_adamw_set_lr(None, 0.1) == st.ST_ERR_INVALID_ARG
    assert lib.st_adamw_read_moments(None, None, None) == st.ST_ERR_INVALID_ARG
    assert lib.st_adamw_write_moments(None, None, None) == st.ST_ERR_INVALID_ARG
    assert lib.st_adamw_step_count(None, None) == st.ST_ERR_INVALID_ARG
    lib.st_adamw_destroy(None)


def test_binding_checks_types_and_sizes(lib):
    p, m = torch.zeros(10), torch.zeros(10)
    with pytest.raises(ValueError):
        st.st_adamw_create([p], [m], [m[:5]], lr=0.1)                       # a moment too short
    with pytest.raises(ValueError):
        st.st_adamw_create([p, p], [m, m], [m], lr=0.1)                     # a list too short
    with pytest.raises(ValueError):
        st.st_adamw_create([p], [m], [m], lr=0.1, weight_decay=[0.1, 0.2])
    with pytest.raises(TypeError):
        st.st_adamw_create([p.double()], [m], [m], lr=0.1)
    with pytest.raises(TypeError):
        st.st_adamw_create([p], [m], [m.double()], lr=0.1)
    with pytest.raises(ValueError):
        st.st_adamw_create([p], [m.to(torch.int8)], [m.to(torch.uint8)], lr=0.1)      # 8 bits without scales
