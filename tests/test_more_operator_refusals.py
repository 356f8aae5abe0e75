"""What layer norm, the embedding and the matrices' steps refuse, on the host alone: no device work is issued here."""
import ctypes as C
import math

import pytest
import torch

from paper_2310_14423_b200 import binding as B
from test_operator_refusals import Placed, Reached, no_library  # noqa: F401


def test_struct_sizes_match_the_header():
    # 5 pointers, 3 int64, 2 int32, 1 double, 3 x (pointer, int64), 3 pointers, 1 int64
    assert C.sizeof(B.QsrLayerNormArgs) == 5 * 8 + 3 * 8 + 8 + 8 + 3 * 16 + 3 * 8 + 8
    # 3 pointers, 5 int64, 2 int32, 1 double, 2 int32, pointer, int64
    assert C.sizeof(B.QsrEmbedArgs) == 3 * 8 + 5 * 8 + 8 + 8 + 8 + 16
    # 4 pointers, 2 int64, 3 int32, 2 floats, 1 int32 | 6 int32, 3 doubles
    assert C.sizeof(B.QsrMatrix) == 4 * 8 + 16 + 24
    assert C.sizeof(B.QsrMuonConfig) == 24 + 24


# ---- layer norm ------------------------------------------------------------------------------------------

def _norm(**kw):
    a = B.QsrLayerNormArgs(x=1 << 20, mean=1 << 21, rstd=1 << 22, rows=4, width=100, x_stride=100, type=0, weight_type=0, eps=1e-5, y=1 << 23, y_stride=100,
                           d_y=1 << 24, d_y_stride=100, d_x=1 << 25, d_x_stride=100, d_weight=1 << 26, d_bias=1 << 27, workspace=1 << 28, workspace_bytes=1 << 20)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_layer_norm_refuses():
    L = B.lib()
    fwd = lambda **kw: L.qsr_layer_norm(C.byref(_norm(**kw)), None)            # noqa: E731
    grad = lambda **kw: L.qsr_layer_norm_grad(C.byref(_norm(**kw)), None)      # noqa: E731
    assert L.qsr_layer_norm(None, None) == B.QSR_EINVAL and L.qsr_layer_norm_grad(None, None) == B.QSR_EINVAL
    assert fwd(rows=0, x=None, y=None) == B.QSR_OK
    both = ((dict(x=None), B.QSR_EINVAL), (dict(type=3), B.QSR_EINVAL), (dict(type=-1), B.QSR_EINVAL), (dict(weight_type=3), B.QSR_EINVAL),
            (dict(rows=-1), B.QSR_ERANGE), (dict(rows=1 << 31), B.QSR_ERANGE), (dict(width=0), B.QSR_ERANGE), (dict(width=(1 << 24) + 1, x_stride=1 << 25), B.QSR_ERANGE),
            (dict(x_stride=99), B.QSR_ERANGE), (dict(x=(1 << 20) + 2), B.QSR_EALIGN), (dict(weight=6), B.QSR_EALIGN), (dict(mean=6), B.QSR_EALIGN),
            (dict(rstd=6), B.QSR_EALIGN))
    for kw, status in both:
        assert fwd(**kw) == status and grad(**kw) == status, kw
    for kw, status in ((dict(y=None), B.QSR_EINVAL), (dict(eps=-1.0), B.QSR_EINVAL), (dict(eps=math.nan), B.QSR_EINVAL), (dict(eps=1e300), B.QSR_EINVAL),
                       (dict(y_stride=99), B.QSR_ERANGE), (dict(y=1 << 20, y_stride=101), B.QSR_ERANGE), (dict(y=(1 << 23) + 2), B.QSR_EALIGN),
                       (dict(bias=6), B.QSR_EALIGN), (dict(y=(1 << 20) + 4), B.QSR_EINVAL), (dict(y=(1 << 20) - 4 * 399), B.QSR_EINVAL)):
        assert fwd(**kw) == status, kw
    for kw, status in ((dict(d_y=None), B.QSR_EINVAL), (dict(mean=None), B.QSR_EINVAL), (dict(rstd=None), B.QSR_EINVAL), (dict(workspace=None), B.QSR_EINVAL),
                       (dict(workspace=(1 << 28) + 128), B.QSR_EALIGN), (dict(workspace_bytes=100), B.QSR_ERANGE), (dict(d_y_stride=99), B.QSR_ERANGE),
                       (dict(d_x_stride=99), B.QSR_ERANGE), (dict(d_y=(1 << 24) + 2), B.QSR_EALIGN), (dict(d_x=(1 << 25) + 2), B.QSR_EALIGN),
                       (dict(d_weight=6), B.QSR_EALIGN), (dict(d_bias=6), B.QSR_EALIGN), (dict(d_x=(1 << 20) + 4), B.QSR_EINVAL),
                       (dict(d_x=(1 << 24) - 4), B.QSR_EINVAL), (dict(d_x=1 << 20, d_x_stride=101), B.QSR_EINVAL)):
        assert grad(**kw) == status, kw
    assert B.qsr_layer_norm_workspace_bytes(10, 10) > 0
    for rows, width in ((-1, 5), (5, 0), (1 << 31, 5), (5, (1 << 24) + 1)):
        with pytest.raises(B.QsrError):
            B.qsr_layer_norm_workspace_bytes(rows, width)


def test_layer_norm_wants_all_tensors_on_the_current_device(no_library):  # noqa: F811
    forward = dict(x=Placed(3, 7), y=Placed(3, 7), weight=Placed(7), bias=Placed(7), mean=Placed(3), rstd=Placed(3))
    grad = dict(x=Placed(3, 7), d_y=Placed(3, 7), mean=Placed(3), rstd=Placed(3), d_x=Placed(3, 7), weight=Placed(7), d_weight=Placed(7), d_bias=Placed(7),
                workspace=Placed(4096, dtype=torch.uint8))
    for call, args in ((B.qsr_layer_norm, forward), (B.qsr_layer_norm_grad, grad)):
        with pytest.raises(Reached):
            call(**args)
        for name, t in args.items():
            with pytest.raises(ValueError):
                call(**{**args, name: Placed(*t.shape, dtype=t.dtype, device=1)})
            if name != "workspace":                 # another type, another size
                with pytest.raises(ValueError):
                    call(**{**args, name: Placed(*t.shape, dtype=torch.float64)})
                with pytest.raises(ValueError):
                    call(**{**args, name: Placed(*(n + 1 for n in t.shape), dtype=t.dtype)})
        with pytest.raises(ValueError):
            call(**{name: Placed(*t.shape, dtype=t.dtype, device=1) for name, t in args.items()})


# ---- embedding -------------------------------------------------------------------------------------------

def _embed(**kw):
    a = B.QsrEmbedArgs(table=1 << 20, tokens=1 << 24, out=1 << 25, rows=4, vocab=50, width=100, table_stride=100, out_stride=100, table_type=0, out_type=0,
                       scale=1.0, workspace=1 << 28, workspace_bytes=1 << 20)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_embedding_refuses():
    L = B.lib()
    fwd = lambda **kw: L.qsr_embed(C.byref(_embed(**kw)), None)            # noqa: E731
    grad = lambda **kw: L.qsr_embed_grad(C.byref(_embed(**kw)), None)      # noqa: E731
    assert L.qsr_embed(None, None) == B.QSR_EINVAL and L.qsr_embed_grad(None, None) == B.QSR_EINVAL
    assert fwd(rows=0, tokens=None, out=None) == B.QSR_OK
    for kw, status in ((dict(table=None), B.QSR_EINVAL), (dict(tokens=None), B.QSR_EINVAL), (dict(out=None), B.QSR_EINVAL), (dict(table_type=3), B.QSR_EINVAL),
                       (dict(out_type=-1), B.QSR_EINVAL), (dict(scale=math.inf), B.QSR_EINVAL), (dict(scale=1e39), B.QSR_EINVAL), (dict(accumulate=2), B.QSR_EINVAL),
                       (dict(reserved=1), B.QSR_EINVAL), (dict(rows=-1), B.QSR_ERANGE), (dict(rows=1 << 31), B.QSR_ERANGE), (dict(vocab=0), B.QSR_ERANGE),
                       (dict(vocab=(1 << 31) - 1), B.QSR_ERANGE), (dict(width=0), B.QSR_ERANGE), (dict(width=(1 << 20) + 1, table_stride=1 << 21, out_stride=1 << 21), B.QSR_ERANGE),
                       (dict(table_stride=99), B.QSR_ERANGE), (dict(out_stride=99), B.QSR_ERANGE), (dict(table=(1 << 20) + 2), B.QSR_EALIGN),
                       (dict(tokens=(1 << 24) + 4), B.QSR_EALIGN), (dict(out=(1 << 25) + 2), B.QSR_EALIGN), (dict(out=(1 << 20) + 4 * 4999), B.QSR_EINVAL),
                       (dict(out=(1 << 20) - 4 * 399), B.QSR_EINVAL)):
        assert fwd(**kw) == status and grad(**kw) == status, kw
    for kw, status in ((dict(workspace=None), B.QSR_EINVAL), (dict(workspace=(1 << 28) + 64), B.QSR_EALIGN), (dict(workspace_bytes=10), B.QSR_ERANGE)):
        assert grad(**kw) == status, kw
    assert 0 < B.qsr_embed_workspace_bytes(10, 10, 10) < B.qsr_embed_workspace_bytes(100000, 10, 1000)
    for args in ((-1, 5, 5), (5, 0, 5), (5, 5, 0), (1 << 31, 5, 5), (5, (1 << 31) - 1, 5), (5, 5, (1 << 20) + 1)):
        with pytest.raises(B.QsrError):
            B.qsr_embed_workspace_bytes(*args)


def test_columns_of_one_buffer_do_not_overlap_by_themselves():
    """A table and its output as different columns of rows of the same stride are accepted; meeting columns are not."""
    at = 1 << 20
    own = dict(table=at, table_stride=300, out_stride=300, rows=0)
    assert B.lib().qsr_embed(C.byref(_embed(**own, out=at + 400)), None) == B.QSR_OK
    for off in (396, 4, 1200 - 396, 1200 + 4):
        assert B.lib().qsr_embed(C.byref(_embed(**{**own, "rows": 4}, out=at + off)), None) == B.QSR_EINVAL


def test_embedding_wants_all_tensors_on_the_current_device(no_library):  # noqa: F811
    i64 = torch.int64
    forward = dict(table=Placed(9, 7), tokens=Placed(3, dtype=i64), out=Placed(3, 7))
    grad = dict(d_out=Placed(3, 7), tokens=Placed(3, dtype=i64), d_table=Placed(9, 7), workspace=Placed(4096, dtype=torch.uint8))
    for call, args in ((B.qsr_embed, forward), (B.qsr_embed_grad, grad)):
        with pytest.raises(Reached):
            call(**args)
        for name, t in args.items():
            with pytest.raises(ValueError):
                call(**{**args, name: Placed(*t.shape, dtype=t.dtype, device=1)})
            if name != "workspace":
                with pytest.raises(ValueError):
                    call(**{**args, name: Placed(*t.shape, dtype=torch.float64)})
        with pytest.raises(ValueError):
            call(**{**args, "tokens": Placed(4, dtype=i64)})
        with pytest.raises(ValueError):
            call(**{name: Placed(*t.shape, dtype=t.dtype, device=1) for name, t in args.items()})


# ---- matrices --------------------------------------------------------------------------------------------

def test_muon_workspace_bytes():
    one, three = B.qsr_muon_workspace_bytes([(100, 2000)], 1, 1), B.qsr_muon_workspace_bytes([(100, 2000)], 1, 3)
    assert 0 < one < three < 2 * one
    assert B.qsr_muon_workspace_bytes([(0, 7)]) > 0
    for shapes, workers, products in (([], 1, 1), ([(5, 5)] * 3, 2, 1), ([(-1, 5)], 1, 1), ([(5, 5)], 0, 1), ([(5, 5)], 1, 2)):
        with pytest.raises(B.QsrError) as e:
            B.qsr_muon_workspace_bytes(shapes, workers, products)
        assert e.value.status == B.QSR_EINVAL
    for shape in ((1, (1 << 20) + 1), (32769, 32769)):
        with pytest.raises(B.QsrError) as e:
            B.qsr_muon_workspace_bytes([shape])
        assert e.value.status == B.QSR_ERANGE


def _muon(change=None, cfg_change=None, n=2, workers=1, workspace=1 << 20, nbytes=1 << 22):
    """Status of qsr_muon_create on made-up addresses that never reach a device: every call here fails a check."""
    t = (B.QsrMatrix * n)()
    for i in range(n):
        base = (1 << 30) + i * (1 << 24)
        t[i] = B.QsrMatrix(param=base, grad=base + (1 << 20), momentum=base + (2 << 20), rows=20, cols=50, param_type=0, grad_type=0, copy_type=B.QSR_NONE,
                           wd_scale=1.0, update_scale=1.0)
    cfg = B.QsrMuonConfig(n_matrices=n, workers=workers, products=1, iterations=5, nesterov=1, beta=0.95, eps=1e-7, weight_decay=0.1)
    if change:
        change(t)
    if cfg_change:
        cfg_change(cfg)
    h = C.c_void_p()
    status = B.lib().qsr_muon_create(C.byref(h), C.byref(cfg), t, workspace, nbytes, None)
    assert not h.value
    return status


def _set(i, **kw):
    def change(t):
        for k, v in kw.items():
            setattr(t[i], k, v)
    return change


def test_muon_create_refuses():
    L = B.lib()
    assert L.qsr_muon_create(None, None, None, None, 0, None) == B.QSR_EINVAL
    for kw, status in ((dict(param=None), B.QSR_EINVAL), (dict(momentum=None), B.QSR_EINVAL), (dict(rows=-1), B.QSR_EINVAL), (dict(param_type=3), B.QSR_EINVAL),
                       (dict(grad_type=B.QSR_NONE), B.QSR_EINVAL), (dict(copy_type=1), B.QSR_EINVAL), (dict(wd_scale=math.nan), B.QSR_EINVAL),
                       (dict(update_scale=math.inf), B.QSR_EINVAL), (dict(reserved=1), B.QSR_EINVAL), (dict(param=(1 << 30) + 2), B.QSR_EALIGN),
                       (dict(grad=(1 << 29) + 1, grad_type=1), B.QSR_EALIGN), (dict(momentum=(1 << 29) + 2), B.QSR_EALIGN),
                       (dict(copy=(1 << 29) + 1, copy_type=2), B.QSR_EALIGN), (dict(rows=40000, cols=40000), B.QSR_ERANGE),
                       # written ranges that meet: the momentum in the parameter, the gradient in it
                       (dict(momentum=(1 << 30) + 3996), B.QSR_EINVAL), (dict(grad=(1 << 30) + 3996), B.QSR_EINVAL)):
        assert _muon(_set(0, **kw)) == status, kw
    assert _muon(_set(1, param=1 << 30)) == B.QSR_EINVAL                     # the same parameter twice
    for name, bad, status in (("workers", 0, B.QSR_EINVAL), ("n_matrices", 0, B.QSR_EINVAL), ("reserved", 1, B.QSR_EINVAL), ("products", 2, B.QSR_EINVAL),
                              ("products", 0, B.QSR_EINVAL), ("nesterov", 2, B.QSR_EINVAL), ("iterations", 0, B.QSR_ERANGE), ("iterations", 17, B.QSR_ERANGE),
                              ("beta", 1.0, B.QSR_EINVAL), ("beta", -0.1, B.QSR_EINVAL), ("beta", math.nan, B.QSR_EINVAL), ("eps", -1e-8, B.QSR_EINVAL),
                              ("eps", math.inf, B.QSR_EINVAL), ("weight_decay", math.nan, B.QSR_EINVAL)):
        assert _muon(cfg_change=lambda c: setattr(c, name, bad)) == status, (name, bad)
    assert _muon(n=3, workers=2) == B.QSR_EINVAL
    assert _muon(_set(1, cols=51), workers=2) == B.QSR_EINVAL                # workers' matrices differ
    assert _muon(_set(1, rows=50, cols=20), workers=2) == B.QSR_EINVAL
    assert _muon(_set(1, param_type=1), workers=2) == B.QSR_EINVAL
    assert _muon(workspace=(1 << 20) + 64) == B.QSR_EALIGN
    assert _muon(nbytes=100) == B.QSR_ERANGE
    assert _muon(workspace=1 << 30) == B.QSR_EINVAL


def test_muon_calls_refuse_null():
    L = B.lib()
    assert L.qsr_muon_destroy(None) == B.QSR_OK
    for status in (L.qsr_muon_step(None, 1e-3, 1.0), L.qsr_muon_sync(None, 0), L.qsr_muon_set_grads(None, None), L.qsr_muon_launch_count(None), L.qsr_muon_check(None)):
        assert status == B.QSR_EINVAL


def test_muon_lists_want_matrices_on_the_current_device(no_library):  # noqa: F811
    def make(change=None, device=0, **other):
        t = lambda name, *s, dtype=torch.float32: Placed(*s, dtype=dtype, device=other.get(name, device))        # noqa: E731
        args = dict(params=[t("first", 30, 20), t("param", 5, 6)], grads=[t("grad", 30, 20), t("grad", 5, 6)], momentum=[t("momentum", 30, 20), t("momentum", 5, 6)],
                    copies=[t("copy", 30, 20, dtype=torch.bfloat16), t("copy", 5, 6, dtype=torch.bfloat16)], workspace=t("workspace", 4096, dtype=torch.uint8))
        B.MuonList(**{**args, **(change or {})})

    with pytest.raises(Reached):
        make()
    for name in ("first", "param", "grad", "momentum", "copy", "workspace"):
        with pytest.raises(ValueError):
            make(**{name: 1})
    with pytest.raises(ValueError):
        make(device=1)
    for change in (dict(params=[Placed(30, 20), Placed(30)]), dict(grads=[Placed(20, 30), Placed(5, 6)]), dict(momentum=[Placed(30, 20, dtype=torch.bfloat16), Placed(5, 6)]),
                   dict(momentum=None), dict(grads=[Placed(30, 20)]), dict(copies=[None]), dict(update_scale=[1.0])):
        with pytest.raises(ValueError):
            make(change)
