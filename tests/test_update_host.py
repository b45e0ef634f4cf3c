"""Weight update and 8-bit calls on the host: refusals before any GPU work, workspace queries, the table's layout."""
import ctypes as C
import math
import os

import pytest

from paper_2311_06837_amd import binding as B
from paper_2311_06837_amd import build as build_mod

P256 = 256      # an address that is never read: every call here is refused, or empty


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        build_mod.build_library()
    return B.lib()


def entry(**kw):
    base = dict(param=P256, grad=P256, m=P256, v=P256, n=10, state_bits=32)
    return B.gnn_param(**{**base, **kw})


def layout(lib, *entries):
    t = (B.gnn_param * max(len(entries), 1))(*entries)
    chunks = C.c_int64(-1)
    return lib.gnn_param_layout(t, len(entries), C.byref(chunks)), t, chunks.value


def test_struct_sizes_are_the_headers():
    assert C.sizeof(B.gnn_param) == B.ParamTable._ROW.size == 7 * 8 + 2 * 8 + 4 * 4
    assert C.sizeof(B.gnn_adamw_hyper) == 4 * 8 + 8 + 8


def test_layout_numbers_the_chunks_through(lib):
    sizes = [1, 0, 1024, 1025, 0, 10 ** 6, 0]
    st, t, chunks = layout(lib, *(entry(n=n) for n in sizes))
    want, at = [], 0
    for n in sizes:
        want.append(at)
        at += -(-n // 1024)
    assert st == 0 and chunks == at and [e.first_chunk for e in t] == want
    assert layout(lib)[0] == 0 and layout(lib)[2] == 0


@pytest.mark.parametrize("status,bad", [
    (1, dict(n=-1)), (1, dict(n=1 << 50)), (4, dict(grad_dtype=2)), (4, dict(param_dtype=7)), (4, dict(state_bits=16)), (1, dict(grad=0)), (1, dict(param=0)),
    (1, dict(m=0)), (1, dict(v=0)), (1, dict(state_bits=8)), (1, dict(state_bits=8, m_scale=P256)), (1, dict(master=P256)), (1, dict(grad=258)),
    (1, dict(param=257, param_dtype=1)), (1, dict(m=258)), (1, dict(weight_decay=math.inf)), (1, dict(weight_decay=math.nan))])
def test_layout_refuses(lib, status, bad):
    assert layout(lib, entry(), entry(**bad))[0] == status
    assert b"tensor 1" in lib.gnn_last_error()


def test_layout_accepts_what_a_tensor_of_the_norm_alone_has(lib):
    assert layout(lib, B.gnn_param(grad=P256 + 2, n=5, grad_dtype=1), B.gnn_param(n=0))[0] == 0
    assert lib.gnn_param_layout(None, 0, None) == 1 and lib.gnn_param_layout(None, 1, C.byref(C.c_int64())) == 1


def test_grad_norm_refuses(lib):
    need = C.c_size_t(0)
    assert lib.gnn_grad_norm(P256, 1, 5, 1.0, 0.0, None, None, C.byref(need), None) == 0 and 5 * 8 <= need.value <= 4096
    assert lib.gnn_grad_norm(P256, 1, 10 ** 9, 1.0, 0.0, None, None, C.byref(need), None) == 0 and need.value <= 1 << 20
    have = C.c_size_t(need.value)
    for args, st in (((P256, -1, 5, 1.0, 0.0, P256), 1), ((P256, 1, -5, 1.0, 0.0, P256), 1), ((None, 1, 5, 1.0, 0.0, P256), 1), ((P256, 0, 5, 1.0, 0.0, P256), 1),
                     ((P256, 1, 5, math.inf, 0.0, P256), 1), ((P256, 1, 5, 1.0, math.nan, P256), 1), ((P256, 1, 5, 1.0, 0.0, None), 1),
                     ((P256, 1, 5, 1.0, 0.0, P256 + 4), 1), ((P256 + 4, 1, 5, 1.0, 0.0, P256), 1)):
        assert lib.gnn_grad_norm(*args, P256, C.byref(have), None) == st, args
    assert lib.gnn_grad_norm(P256, 1, 5, 1.0, 0.0, P256, None, None, None) == 1
    assert lib.gnn_grad_norm(P256, 1, 5, 1.0, 0.0, P256, P256, C.byref(C.c_size_t(8)), None) == 3
    assert lib.gnn_grad_norm(P256, 1, 5, 1.0, 0.0, P256, P256 + 8, C.byref(have), None) == 1


@pytest.mark.parametrize("bad", [dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0),
                                 dict(eps=1e-60), dict(eps=math.inf), dict(step=0), dict(grad_scale=math.nan)])
def test_adamw_refuses(lib, bad):
    h = B.gnn_adamw_hyper(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, grad_scale=1.0), **bad})
    assert lib.gnn_adamw_step(P256, 1, 1, C.byref(h), None, None, None) == 1


@pytest.mark.parametrize("eps,status", [(1e-40, 1), (1.1e-38, 1), (1e-30, 1), (1e-18, 1), (9.9e-17, 1), (1.1e30, 1), (-1e-8, 1), (math.nan, 1),
                                        (1e-16, 0), (1e-15, 0), (1e-8, 0), (1.0, 0), (1e30, 0)])
def test_adamw_takes_an_eps_that_floats_can_divide_by(lib, eps, status):
    """Below 2.9e-39 the reciprocal of eps is infinite and a weight with zero moments became NaN; below the root of the smallest second
    moment that is kept the step of a weight with tiny gradients was m / eps.  No tensors: an accepted call does nothing."""
    h = B.gnn_adamw_hyper(lr=1e-3, beta1=0.9, beta2=0.999, eps=eps, step=1, grad_scale=1.0)
    assert lib.gnn_adamw_step(None, 0, 0, C.byref(h), None, None, None) == status
    assert status == 0 or b"eps" in lib.gnn_last_error()


@pytest.mark.parametrize("lr,beta1,status", [(1e39, 0.0, 1), (1e38, 0.9, 1), (math.inf, 0.9, 1), (math.nan, 0.9, 1), (-1e-9, 0.9, 1), (1e37, 0.9, 0), (0.0, 0.9, 0)])
def test_adamw_takes_a_rate_whose_first_step_is_a_float(lib, lr, beta1, status):
    """An infinite lr / (1 - beta1) times the zero update of a weight that nothing has reached was NaN."""
    h = B.gnn_adamw_hyper(lr=lr, beta1=beta1, beta2=0.999, eps=1e-8, step=1, grad_scale=1.0)
    assert lib.gnn_adamw_step(None, 0, 0, C.byref(h), None, None, None) == status
    assert status == 0 or b"lr" in lib.gnn_last_error()


def test_adamw_refuses_tables(lib):
    h = B.gnn_adamw_hyper(1e-3, 0.9, 0.999, 1e-8, 1, 1.0)
    assert lib.gnn_adamw_step(P256, 1, 1, None, None, None, None) == 1
    assert lib.gnn_adamw_step(None, 1, 1, C.byref(h), None, None, None) == 1
    assert lib.gnn_adamw_step(P256, 1, 1, C.byref(h), None, P256 + 4, None) == 1
    assert lib.gnn_adamw_step(None, 0, 0, C.byref(h), None, None, None) == 0     # no tensors: nothing to do


def test_state_values_refuses(lib):
    assert lib.gnn_adamw_state_values(None, None, None, None, 0, None, None, 0, None) == 0
    assert lib.gnn_adamw_state_values(None, P256, P256, P256, 5, P256, P256, 0, None) == 1
    assert lib.gnn_adamw_state_values(P256, P256, P256, P256, -1, P256, P256, 0, None) == 1
    assert lib.gnn_adamw_state_values(P256, P256, P256, P256, 5, P256, P256, 2, None) == 4


def test_quantize_rows_refuses(lib):
    good = dict(rows=None, n=3, X=P256, ldx=20, K=20, dtype=0, Q=P256, ldq=32, scale=P256, values=None, ldv=0)
    call = lambda **kw: lib.gnn_quantize_rows(*{**good, **kw}.values(), None)
    for st, bad in ((1, dict(n=-1)), (4, dict(dtype=2)), (1, dict(K=0)), (4, dict(K=65537, ldx=65537, ldq=65552)), (2, dict(ldx=19)), (2, dict(ldq=16)), (2, dict(ldq=40)),
                    (2, dict(values=P256, ldv=19)), (1, dict(X=None)), (1, dict(Q=None)), (1, dict(scale=None)), (1, dict(Q=P256 + 8))):
        assert call(**bad) == st, bad
    assert call(n=0, X=None, Q=None, scale=None) == 0


def test_quantize_weight_refuses(lib):
    need = C.c_size_t(0)
    good = dict(W=P256, ldw=7, K=300, N=7, dtype=1, Wq=P256, scale=P256, values=None, ldv=0, ws=P256)
    call = lambda have=1 << 20, **kw: lib.gnn_quantize_weight(*{**good, **kw}.values(), C.byref(C.c_size_t(have)), None)
    for st, bad in ((4, dict(dtype=2)), (1, dict(K=0)), (1, dict(N=0)), (4, dict(K=70000)), (4, dict(N=70000, ldw=70000)), (2, dict(ldw=6)), (2, dict(values=P256, ldv=6)),
                    (1, dict(W=None)), (1, dict(Wq=None)), (1, dict(scale=None)), (1, dict(Wq=P256 + 8)), (1, dict(ws=P256 + 8)), (3, dict(have=16))):
        assert call(**bad) == st, bad
    assert lib.gnn_quantize_weight(None, 7, 300, 7, 1, None, None, None, 0, None, C.byref(need), None) == 0 and need.value >= 7 * 4


def test_linear_i8_refuses(lib):
    good = dict(rows=None, n=3, A=P256, sa=P256, X=P256, sx=P256, ld=32, K=20, dt=2, Wn=P256, wn=P256, Ws=P256, ws_=P256, bias=None, N=9, H=P256, ldh=9, relu=0, out=0, ws=P256)
    call = lambda have=1 << 20, **kw: lib.gnn_linear_i8_fwd(*{**good, **kw}.values(), C.byref(C.c_size_t(have)), None)
    for st, bad in ((1, dict(n=-1)), (4, dict(dt=3)), (4, dict(out=2)), (1, dict(K=0)), (1, dict(N=0)), (4, dict(K=65537, ld=65552)), (4, dict(N=65537, ldh=65537)),
                    (2, dict(ld=16)), (2, dict(ld=24)), (2, dict(ldh=8)), (1, dict(X=None)), (1, dict(Ws=None)), (1, dict(A=None)), (1, dict(Wn=None)), (1, dict(wn=None)),
                    (1, dict(ws_=None)), (1, dict(H=None)), (1, dict(sa=None)), (1, dict(sx=None)), (1, dict(A=P256 + 8)), (1, dict(X=P256 + 8)), (1, dict(Wn=P256 + 8)),
                    (1, dict(Ws=P256 + 8)), (3, dict(dt=0, have=8, K=2000, ld=2000)), (1, dict(ws=P256 + 8))):
        assert call(**bad) == st, bad
    assert call(n=0, A=None, sa=None, X=P256, H=None) == 0
    need = C.c_size_t(0)
    args = [*{**good, **dict(dt=1, n=1000)}.values()][:-1]
    assert lib.gnn_linear_i8_fwd(*args, None, C.byref(need), None) == 0


def test_product_refuses_codes_that_end_inside_a_group_of_sixteen():
    """The kernels read codes in groups of 16 columns: a matrix of X_self that ends at K may end inside the last one."""
    torch = pytest.importorskip("torch")
    w = B.Int8Weight(torch.zeros(B.Int8Weight.bytes(20, 9), dtype=torch.int8), torch.zeros(9), 20, 9)
    A, s, H = torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3), torch.zeros(3, 9)
    X = torch.zeros(2 * 32 + 20, dtype=torch.int8).as_strided((3, 20), (32, 1))
    with pytest.raises(AssertionError, match="X_self"):
        B.gnn_linear_i8_fwd(None, 3, A, s, X, s, 20, w, w, None, H, False)


def test_table_refuses_tensors_it_cannot_read():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="grad"):
        B.ParamTable([{"grad": torch.zeros(4)}])          # on the host
    with pytest.raises(ValueError, match="unknown"):
        B.ParamTable([{"grad": torch.zeros(4), "momentum": torch.zeros(4)}])
