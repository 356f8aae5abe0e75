"""What the tensor lists and the token log probabilities refuse, on the host alone: no device work is issued here."""
import ctypes as C
import math

import pytest
import torch

from paper_2310_14423_b200 import binding as B


def test_struct_sizes_match_the_header():
    # 7 pointers, 1 int64, 3 int32 + float | 4 int32, 5 doubles, 1 pointer | see the header
    assert C.sizeof(B.QsrTensor) == 7 * 8 + 8 + 16
    assert C.sizeof(B.QsrListConfig) == 16 + 40 + 8
    assert C.sizeof(B.QsrLogprobArgs) == 2 * 8 + 3 * 8 + 8 + 8 + 8 * 8 + 8


def test_list_workspace_bytes():
    assert B.qsr_list_workspace_bytes([10]) > 0
    assert B.qsr_list_workspace_bytes([0]) > 0
    small, large = B.qsr_list_workspace_bytes([1000] * 6, 3), B.qsr_list_workspace_bytes([100_000_000] * 6, 3)
    assert 0 < small < large < 100_000_000
    for numels, workers in (([], 1), ([5, 5, 5], 2), ([-1], 1), ([5], 0)):
        with pytest.raises(B.QsrError) as e:
            B.qsr_list_workspace_bytes(numels, workers)
        assert e.value.status == B.QSR_EINVAL


def _list(change=None, cfg_change=None, n=2, workers=1, workspace=1 << 20, nbytes=1 << 20):
    """Status of qsr_list_create on made-up addresses that never reach a device: every call here fails a check."""
    t = (B.QsrTensor * n)()
    for i in range(n):
        base = (1 << 30) + i * (1 << 24)
        t[i] = B.QsrTensor(param=base, grad=base + (1 << 20), m=base + (2 << 20), v=base + (3 << 20), numel=1000, param_type=0, grad_type=0,
                           copy_type=B.QSR_NONE, wd_scale=1.0)
    cfg = B.QsrListConfig(n_tensors=n, workers=workers, states=0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
    if change:
        change(t)
    if cfg_change:
        cfg_change(cfg)
    h = C.c_void_p()
    status = B.lib().qsr_list_create(C.byref(h), C.byref(cfg), t, workspace, nbytes, None)
    assert not h.value
    return status


def _set(i, **kw):
    def change(t):
        for k, v in kw.items():
            setattr(t[i], k, v)
    return change


def test_list_create_refuses():
    L = B.lib()
    assert L.qsr_list_create(None, None, None, None, 0, None) == B.QSR_EINVAL
    assert _list(_set(0, param=None)) == B.QSR_EINVAL
    assert _list(_set(0, m=None)) == B.QSR_EINVAL
    assert _list(_set(1, v=None)) == B.QSR_EINVAL
    assert _list(_set(0, numel=-1)) == B.QSR_EINVAL
    assert _list(_set(0, param_type=3)) == B.QSR_EINVAL
    assert _list(_set(0, grad_type=B.QSR_NONE)) == B.QSR_EINVAL
    assert _list(_set(0, copy_type=1)) == B.QSR_EINVAL                       # a copy without an address
    assert _list(_set(0, wd_scale=math.nan)) == B.QSR_EINVAL
    assert _list(_set(0, param=(1 << 30) + 2)) == B.QSR_EALIGN
    assert _list(_set(0, grad=(1 << 29) + 1, grad_type=1)) == B.QSR_EALIGN
    assert _list(_set(0, m=(1 << 29) + 2)) == B.QSR_EALIGN
    assert _list(cfg_change=lambda c: setattr(c, "states", 1)) == B.QSR_EINVAL   # no scales
    assert _list(cfg_change=lambda c: setattr(c, "states", 2)) == B.QSR_EINVAL
    assert _list(cfg_change=lambda c: setattr(c, "workers", 0)) == B.QSR_EINVAL
    assert _list(cfg_change=lambda c: setattr(c, "n_tensors", 0)) == B.QSR_EINVAL
    assert _list(cfg_change=lambda c: setattr(c, "reserved", 1)) == B.QSR_EINVAL
    for name, bad in (("beta1", 1.0), ("beta1", -0.1), ("beta2", math.nan), ("eps", -1e-8), ("eps", math.inf), ("weight_decay", math.inf)):
        assert _list(cfg_change=lambda c, n=name, b=bad: setattr(c, n, b)) == B.QSR_EINVAL, (name, bad)
    assert _list(n=3, workers=2) == B.QSR_EINVAL
    assert _list(_set(1, numel=999), workers=2) == B.QSR_EINVAL              # workers' tensors differ
    assert _list(_set(1, param_type=1), workers=2) == B.QSR_EINVAL
    assert _list(workspace=(1 << 20) + 64) == B.QSR_EALIGN
    assert _list(nbytes=100) == B.QSR_ERANGE
    # written ranges that meet: the same parameter twice, m inside v, the gradient inside the parameter, the workspace
    assert _list(_set(1, param=1 << 30)) == B.QSR_EINVAL
    assert _list(_set(0, m=(1 << 30) + (3 << 20) + 3996)) == B.QSR_EINVAL
    assert _list(_set(0, grad=(1 << 30) + 3996)) == B.QSR_EINVAL
    assert _list(workspace=1 << 30) == B.QSR_EINVAL


def test_list_calls_refuse_null():
    L = B.lib()
    assert L.qsr_list_destroy(None) == B.QSR_OK
    assert L.qsr_list_step(None, 1, 1e-3, 1.0) == B.QSR_EINVAL
    assert L.qsr_list_sync(None, 0) == B.QSR_EINVAL
    assert L.qsr_list_set_grads(None, None) == B.QSR_EINVAL
    assert L.qsr_list_launch_count(None) == B.QSR_EINVAL


def _args(**kw):
    a = B.QsrLogprobArgs(logits=1 << 20, tokens=1 << 21, rows=4, vocab=100, row_stride=100, logits_type=0, n_top=0, inv_temperature=1.0,
                         logprob=1 << 22)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_logprob_calls_refuse():
    L = B.lib()
    fwd = lambda **kw: L.qsr_token_logprobs(C.byref(_args(**kw)), None)            # noqa: E731
    grad = lambda **kw: L.qsr_token_logprobs_grad(C.byref(_args(**{**dict(d_logits=1 << 23, d_row_stride=100, row_stats=1 << 24), **kw})), None)  # noqa: E731
    assert L.qsr_token_logprobs(None, None) == B.QSR_EINVAL and L.qsr_token_logprobs_grad(None, None) == B.QSR_EINVAL
    assert fwd(rows=0, logits=None, tokens=None, logprob=None) == B.QSR_OK
    for kw in (dict(logits=None), dict(tokens=None), dict(logprob=None), dict(logits_type=3), dict(logits_type=-1), dict(inv_temperature=0.0),
               dict(inv_temperature=-1.0), dict(inv_temperature=math.nan), dict(inv_temperature=1e300), dict(n_top=3)):
        assert fwd(**kw) == B.QSR_EINVAL, kw
    for kw in (dict(rows=-1), dict(rows=1 << 28), dict(vocab=0), dict(vocab=1 << 31, row_stride=1 << 31), dict(row_stride=99),
               dict(n_top=-1), dict(n_top=33), dict(n_top=5, vocab=4), dict(d_logits=1 << 23, d_row_stride=99),
               dict(d_logits=1 << 20, d_row_stride=101)):
        assert fwd(**kw) == B.QSR_ERANGE, kw
    for kw in (dict(logits=(1 << 20) + 2), dict(tokens=(1 << 21) + 4), dict(logprob=(1 << 22) + 2), dict(entropy=1 << 22 | 2), dict(row_stats=(1 << 22) + 4),
               dict(n_top=2, top_logprob=(1 << 24) + 2, top_token=1 << 25), dict(n_top=2, top_logprob=1 << 24, top_token=(1 << 25) + 4),
               dict(d_logprob=(1 << 22) + 1), dict(d_entropy=(1 << 22) + 1), dict(d_logits=(1 << 23) + 2, d_row_stride=100)):
        assert fwd(**kw) == B.QSR_EALIGN, kw
    assert grad(d_logits=None) == B.QSR_EINVAL
    assert grad(row_stats=None) == B.QSR_EINVAL
    assert grad(d_entropy=1 << 25) == B.QSR_EINVAL


class Placed:
    """What the binding asks of a tensor, for one that lies on a device of this index at an address that nothing reads."""

    def __init__(self, *shape, dtype=torch.float32, device=0):
        self.shape, self.dtype, self.index, self.device = torch.Size(shape), dtype, device, torch.device("cuda", device)
        self.is_cuda = True

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def data_ptr(self):
        return 1 << 30


class Reached(Exception):
    pass


@pytest.fixture
def no_library(monkeypatch):
    """Every argument has passed when the library is asked for."""
    def reached():
        raise Reached
    monkeypatch.setattr(B, "lib", reached)
    monkeypatch.setattr(B, "_current_device", lambda: 0, raising=False)


def test_lists_want_all_tensors_on_the_current_device(no_library):
    def make(states, **other):
        """A list of two tensors, some of its operands on device 1."""
        t = lambda n, name, dtype=torch.float32: Placed(n, dtype=dtype, device=other.get(name, 0))        # noqa: E731
        f8 = torch.float8_e4m3fn if states == "e4m3" else torch.float32
        scale = lambda name: [t(2, name), t(1, name)] if states == "e4m3" else None                        # noqa: E731
        B.TensorList([t(300, "first"), t(5, "param")], [t(300, "grad"), t(5, "grad")], [t(300, "m", f8), t(5, "m", f8)],
                     [t(300, "v", f8), t(5, "v", f8)], m_scale=scale("m_scale"), v_scale=scale("v_scale"),
                     copies=[t(300, "copy", torch.bfloat16), t(5, "copy", torch.bfloat16)], grad_norm=t(1, "grad_norm"),
                     workspace=t(4096, "workspace", torch.uint8))

    for states in ("f32", "e4m3"):
        with pytest.raises(Reached):
            make(states)
        for name in ("first", "param", "grad", "m", "v", "copy", "grad_norm", "workspace") + (("m_scale", "v_scale") if states == "e4m3" else ()):
            with pytest.raises(ValueError):
                make(states, **{name: 1})
        with pytest.raises(ValueError):       # all of them on a device that is not the current one
            make(states, first=1, param=1, grad=1, m=1, v=1, copy=1, grad_norm=1, workspace=1, m_scale=1, v_scale=1)


def test_log_probabilities_want_all_tensors_on_the_current_device(no_library):
    i64 = torch.int64
    own = dict(logits=Placed(3, 7), tokens=Placed(3, dtype=i64))
    forward = dict(own, logprob=Placed(3), entropy=Placed(3), row_stats=Placed(3, 2), top_logprob=Placed(3, 2), top_token=Placed(3, 2, dtype=i64),
                   d_logprob=Placed(3), d_entropy=Placed(3), d_logits=Placed(3, 7))
    grad = dict(own, row_stats=Placed(3, 2), d_logits=Placed(3, 7), d_logprob=Placed(3), d_entropy=Placed(3), entropy=Placed(3))
    for call, args in ((B.qsr_token_logprobs, forward), (B.qsr_token_logprobs_grad, grad)):
        with pytest.raises(Reached):
            call(**args)
        for name, t in args.items():
            with pytest.raises(ValueError):
                call(**{**args, name: Placed(*t.shape, dtype=t.dtype, device=1)})
        with pytest.raises(ValueError):
            call(**{name: Placed(*t.shape, dtype=t.dtype, device=1) for name, t in args.items()})


def test_gradients_that_overlap_the_logits_without_being_them():
    """fp32 logits of 4 x 100 at 2^20, rows 100 or 250 apart.  Accepted layouts are tested on the GPU."""
    at = 1 << 20
    for kw in (dict(d_logits=at + 4), dict(d_logits=at - 4), dict(d_logits=at + 4 * 399), dict(d_logits=at - 4 * 399),
               dict(d_logits=at + 4 * 100), dict(d_logits=at, d_row_stride=100, row_stride=100, logits=at + 40),
               dict(row_stride=250, d_row_stride=250, d_logits=at + 4 * 99), dict(row_stride=250, d_row_stride=250, d_logits=at + 4 * 151),
               dict(row_stride=250, d_row_stride=250, d_logits=at - 4 * (250 + 99)), dict(row_stride=250, d_row_stride=250, d_logits=at + 4 * (750 + 99)),
               dict(row_stride=250, d_row_stride=251, d_logits=at + 4 * 100), dict(row_stride=1 << 62, d_row_stride=1 << 62, d_logits=at + 4),
               dict(rows=1, d_logits=at + 4 * 99), dict(rows=1, row_stride=500, d_row_stride=600, d_logits=at - 4 * 99)):
        args = {**dict(d_row_stride=100, row_stats=1 << 24), **kw}
        assert B.lib().qsr_token_logprobs(C.byref(_args(**args)), None) == B.QSR_EINVAL, kw
        assert B.lib().qsr_token_logprobs_grad(C.byref(_args(**args)), None) == B.QSR_EINVAL, kw


def test_temperatures_whose_base_two_factor_overflows():
    """exp(tau z) is 2^(c z) with c = tau log2(e), which has to be finite in fp32."""
    for tau in (2.5e38, 3.4e38):
        assert B.lib().qsr_token_logprobs(C.byref(_args(inv_temperature=tau)), None) == B.QSR_EINVAL
        assert B.lib().qsr_token_logprobs(C.byref(_args(inv_temperature=tau, rows=0)), None) == B.QSR_EINVAL
    assert B.lib().qsr_token_logprobs(C.byref(_args(inv_temperature=2e38, rows=0)), None) == B.QSR_OK
