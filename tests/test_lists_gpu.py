"""Tensor lists on the GPU -- AdamW steps with states in 32 and 8 bits, clipping, replica means -- against the formulas of
include/qsr.h in binary64 (numpy).  Tolerances are sums of the roundings each quantity goes through (u = 2^-24)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2310_14423_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # relative, of a normal number
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}       # absolute, below the smallest normal one
SIZES = [1, 2, 7, 8, 9, 31, 32, 33, 255, 256, 257, 511, 777, 2047, 2048, 2049, 4100, 0, 8192, 8200, 20003]
CODES = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()     # the format's 256 values
CANARY = 77.0


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Lists:
    """Tensors of `sizes` for K workers cut out of guarded flat buffers, `lead` elements apart, on the GPU and as numpy."""

    def __init__(self, sizes, K=1, param="f32", grad="f32", copy=None, states="f32", lead=64, seed=0, n_old=5, **kw):
        self.sizes, self.K, self.types, self.states = list(sizes), K, (param, grad, copy), states
        rng = np.random.default_rng(seed)
        self.n = len(self.sizes) * K
        every = self.sizes * K
        mag = [2.0 ** rng.uniform(-14, 0) for _ in every]
        self.buffers = []
        self.p = self._cut([rng.normal(0, 0.5, n) for n in every], T[param], lead)
        self.g = self._cut([rng.normal(0, 1, n) * s for n, s in zip(every, mag)], T[grad], lead)
        self.c = self._cut([np.zeros(n) for n in every], T[copy], lead) if copy else None
        m = [rng.normal(0, 0.3, n) * s * (n_old > 0) for n, s in zip(every, mag)]
        u = [np.abs(rng.normal(0.8, 0.3, n)) * s * (n_old > 0) for n, s in zip(every, mag)]
        if states == "f32":
            self.m, self.v = self._cut(m, torch.float32, lead), self._cut([x * x for x in u], torch.float32, lead)
            self.ms = self.vs = None
        else:
            codes_m, codes_u = [quantise(x.astype(np.float32), False) for x in m], [quantise(x.astype(np.float32), True) for x in u]
            f8 = torch.float8_e4m3fn
            self.m, self.v = self._cut([c for c, _ in codes_m], f8, lead), self._cut([c for c, _ in codes_u], f8, lead)
            self.ms, self.vs = self._cut([s for _, s in codes_m], torch.float32, 3), self._cut([s for _, s in codes_u], torch.float32, 3)
        self.workspace = torch.full((B.qsr_list_workspace_bytes(every, K),), 255, dtype=torch.uint8, device=DEV)
        self.wd = [float(x) for x in rng.choice([0.0, 0.5, 1.0], len(every))]
        self.list = B.TensorList(self.p, self.g, self.m, self.v, m_scale=self.ms, v_scale=self.vs, copies=self.c, wd_scale=self.wd,
                                 workers=K, workspace=self.workspace, stream=_stream(), **kw)
        self.before = self.numpy()

    def _cut(self, arrays, dtype, lead):
        total = sum(a.size + lead for a in arrays) + lead
        flat = torch.full((total,), CANARY, device=DEV).to(dtype)
        at, out, used = lead, [], torch.zeros(total, dtype=torch.bool, device=DEV)
        for a in arrays:
            x = flat[at:at + a.size]
            x.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(DEV).float().to(dtype))
            used[at:at + a.size] = True
            out.append(x)
            at += a.size + lead
        self.buffers.append((flat, used))
        return out

    def numpy(self):
        def host(xs):
            return None if xs is None else [x.double().cpu().numpy() for x in xs]
        return {"p": host(self.p), "g": host(self.g), "c": host(self.c), "m": host(self.m), "v": host(self.v), "ms": host(self.ms), "vs": host(self.vs)}

    def assert_guards(self):
        for flat, used in self.buffers:
            assert bool((flat.float()[~used] == torch.tensor(CANARY).to(flat.dtype).float().item()).all())


def blocks(x):
    """x padded with zeros to whole blocks of 256, [blocks, 256]."""
    return np.concatenate([x, np.zeros((-x.size) % 256, x.dtype)]).reshape(-1, 256)


def nearest_code(q):
    """Nearest E4M3 value, ties to the even code (numpy, any float)."""
    pos = CODES[:127]                                    # 0 .. 448
    a = np.minimum(np.abs(np.asarray(q, np.float64)), 448.0)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    up = (a - pos[lo] > pos[hi] - a) | ((a - pos[lo] == pos[hi] - a) & (hi % 2 == 0))
    return np.copysign(np.where(up, pos[hi], pos[lo]), q)


def quantise(x32, positive):
    """(codes, scales) of a fp32 array by the format's definition, every operation one fp32 rounding."""
    b = blocks(x32)
    amax = np.abs(b).max(1, initial=0).astype(np.float32)
    scale = np.where(amax >= np.float32(2.0 ** -100), amax * np.float32(1.0 / 448.0), np.float32(0)).astype(np.float32)
    with np.errstate(divide="ignore"):
        inv = np.where(scale > 0, np.float32(1) / scale, np.float32(0)).astype(np.float32)
    q = (b * inv[:, None]).astype(np.float32)
    if positive:
        q = np.where(q > 0, np.maximum(q, np.float32(2.0 ** -9)), q)
    return nearest_code(q).reshape(-1)[:x32.size], scale


def dequantise(codes, scale):
    return (blocks(codes) * scale[:, None]).reshape(-1)[:codes.size]


def expected(L, n, lr, wd, grad_scale=1.0, clip=0.0, beta1=0.9, beta2=0.999, eps=1e-8):
    """Per tensor: (theta, m, v) in binary64 and the error bounds of theta, m and v in fp32."""
    b, out = L.before, []
    T_ = len(L.sizes)
    for k in range(L.K):
        scaled = [grad_scale * g for g in b["g"][k * T_:(k + 1) * T_]]
        norm = math.sqrt(sum(float((g * g).sum()) for g in scaled))
        f = min(1.0, clip / (norm + 1e-6)) if clip > 0 else 1.0
        for j in range(T_):
            i = k * T_ + j
            g, th = scaled[j] * f, b["p"][i]
            if L.states == "f32":
                m0, v0 = b["m"][i], b["v"][i]
            else:
                m0, v0 = dequantise(b["m"][i], b["ms"][i]), dequantise(b["v"][i], b["vs"][i]) ** 2
            m, v = beta1 * m0 + (1 - beta1) * g, beta2 * v0 + (1 - beta2) * g * g
            d = np.sqrt(v) / math.sqrt(1 - beta2 ** n) + eps
            up = lr / (1 - beta1 ** n) * m / d
            th1 = th - (lr * wd * L.wd[i] * th + up)
            # the gradient: one rounding for the scale, and with clipping the factor's own error (a sum over all elements)
            eg = (2 + (64 if clip > 0 else 0)) * U
            em = (4 * U) * (np.abs(m0) + np.abs(g)) + eg * np.abs(g)
            ev = (6 * U) * (v0 + g * g) + 2 * eg * g * g
            # root (2 ulp), scaling, sum, reciprocal (2 ulp), two products: 10 roundings of the update; the decay, two
            # sums, and the final rounding
            eup = lr / (1 - beta1 ** n) / d * em + np.abs(up) * (10 * U + ev / np.maximum(2 * v, 1e-300))
            eth = eup + 4 * U * (np.abs(lr * wd * th) + np.abs(up)) + U * np.abs(th1)
            out.append((th1, m, v, eth, em, ev))
    return out


def check_step(L, want, n_rounds=1):
    got = L.numpy()
    param, grad, copy = L.types
    for i, (th, m, v, eth, em, ev) in enumerate(want):
        if th.size == 0:
            continue
        tol = eth + HALF_ULP[param] * (np.abs(th) + eth) * (param != "f32") + TINY[param]
        assert np.all(np.abs(got["p"][i] - th) <= tol), (i, th.size, np.max(np.abs(got["p"][i] - th) / tol))
        if copy:
            tol = eth + HALF_ULP[copy] * (np.abs(th) + eth) * (copy != "f32") + TINY[copy]
            assert np.all(np.abs(got["c"][i] - th) <= tol)
        if L.states == "f32":
            assert np.all(np.abs(got["m"][i] - m) <= em + 1e-44), (i, np.max(np.abs(got["m"][i] - m) / np.maximum(em, 1e-300)))
            assert np.all(np.abs(got["v"][i] - v) <= ev + 1e-44), (i, np.max(np.abs(got["v"][i] - v) / np.maximum(ev, 1e-300)))
        else:
            for x, e, codes, scale in ((m, em, got["m"][i], got["ms"][i]),
                                       (np.sqrt(v), ev / np.maximum(2 * np.sqrt(v), 1e-300) + U * np.sqrt(v), got["v"][i], got["vs"][i])):
                amax = np.abs(blocks(x)).max(1)
                assert np.all(np.abs(scale - amax / 448.0) <= (blocks(e).max(1) / 448.0 + 2 * U * amax / 448.0))
                # half a step of three mantissa bits, or half the smallest step (the whole one where 0 is not allowed)
                s = np.repeat(scale, 256)[:x.size]
                tol = e + np.abs(x) * (2.0 ** -4 + 8 * U) + s * 2.0 ** -9
                assert np.all(np.abs(codes * s - x) <= tol)
    L.assert_guards()


TYPES = [("f32", "f32", None), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("bf16", "bf16", None), ("f16", "f16", None), ("bf16", "f32", None)]


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("lead", [64, 1, 3, 8])
@pytest.mark.parametrize("types", TYPES, ids=["-".join(str(x) for x in t) for t in TYPES])
def test_step_matches_the_formula(types, lead, states):
    param, grad, copy = types
    L = Lists(SIZES, param=param, grad=grad, copy=copy, states=states, lead=lead, weight_decay=0.1, seed=lead)
    L.list.qsr_list_step(6, 1e-2)
    check_step(L, expected(L, 6, 1e-2, 0.1))
    assert L.list.qsr_list_launch_count() == 1


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_first_step_from_zero_states(states):
    L = Lists([5, 256, 3000], states=states, n_old=0, weight_decay=0.0)
    L.list.qsr_list_step(1, 1e-3)
    check_step(L, expected(L, 1, 1e-3, 0.0))


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("clip", [1e-3, 0.5, 1e6])
def test_clipping_is_per_worker(clip, states):
    norms = torch.zeros(3, device=DEV)
    L = Lists([300, 7, 5000, 256], K=3, grad="bf16", states=states, lead=5, clip_norm=clip, grad_norm=norms, weight_decay=0.05, seed=3)
    L.list.qsr_list_step(4, 1e-3, 0.25)
    check_step(L, expected(L, 4, 1e-3, 0.05, grad_scale=0.25, clip=clip))
    want = [math.sqrt(sum(float((0.0625 * g * g).sum()) for g in L.before["g"][4 * k:4 * k + 4])) for k in range(3)]
    assert np.allclose(norms.cpu().numpy(), want, rtol=64 * U, atol=0)
    assert L.list.qsr_list_launch_count() == 2
    first = L.numpy()["p"]
    again = Lists([300, 7, 5000, 256], K=3, grad="bf16", states=states, lead=5, clip_norm=clip, weight_decay=0.05, seed=3)
    again.list.qsr_list_step(4, 1e-3, 0.25)
    assert all(np.array_equal(a, b) for a, b in zip(first, again.numpy()["p"]))       # the same bits every time


def test_codes_are_a_function_of_the_formulas_alone():
    """Twenty steps with 8-bit states: codes and scales equal a numpy restatement in fp32, operation by operation, bit for bit."""
    L = Lists([256 * 9, 1000, 33, 5], states="e4m3", grad="bf16", n_old=0, weight_decay=0.01)
    omb1, omb2, f = np.float32(1 - 0.9), np.float32(1 - 0.999), np.float32
    ref = [(np.zeros(n, f), np.zeros(n, f)) for n in L.sizes]
    rng = np.random.default_rng(8)
    for step in range(1, 21):
        for i, n in enumerate(L.sizes):
            L.g[i].copy_(torch.from_numpy(rng.normal(0, 10.0 ** rng.uniform(-6, 0), n)).to(DEV).to(torch.bfloat16))
        L.list.qsr_list_step(step, 1e-3)
        got = L.numpy()
        for i in range(len(L.sizes)):
            g = got["g"][i].astype(f)
            m, u = ref[i]
            v = u * u
            m = m + omb1 * (g - m)
            u = np.sqrt(v + omb2 * (g * g - v))
            cm, sm = quantise(m, False)
            cu, su = quantise(u, True)
            assert np.array_equal(got["ms"][i], sm.astype(np.float64)) and np.array_equal(got["vs"][i], su.astype(np.float64)), (step, i)
            assert np.array_equal(got["m"][i], cm) and np.array_equal(got["v"][i], cu), (step, i)
            ref[i] = (dequantise(cm.astype(f), sm).astype(f), dequantise(cu.astype(f), su).astype(f))
    assert any((c > 0).all() for c in got["v"])           # nothing that was positive became zero


def test_e4m3_training_follows_fp32_states():
    """A quadratic: with 8-bit states the loss falls like with fp32 states."""
    loss = {}
    for states in ("f32", "e4m3"):
        L = Lists([4096, 700], states=states, n_old=0, seed=4)
        rng = np.random.default_rng(1)
        target = [torch.from_numpy(rng.normal(0, 1, n)).to(DEV).float() for n in L.sizes]
        lam = [torch.from_numpy(10.0 ** rng.uniform(-3, 0, n)).to(DEV).float() for n in L.sizes]
        for n in range(1, 301):
            for p, g, t, l in zip(L.p, L.g, target, lam):
                g.copy_(l * (p - t))
            L.list.qsr_list_step(n, 2e-2)
        loss[states] = sum(float((l * (p - t).square()).sum()) for p, t, l in zip(L.p, target, lam))
    start = sum(float((l * (torch.from_numpy(p).to(DEV) - t).square()).sum()) for p, t, l in zip(L.before["p"], target, lam))
    assert loss["f32"] < 0.05 * start and loss["e4m3"] < 0.05 * start


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_nan_and_infinity_stay_in_their_element(states):
    L = Lists([1000, 300], states=states, weight_decay=0.1)
    L.g[0][300] = math.nan
    L.g[0][900] = math.inf
    L.g[1][7] = -math.inf
    L.before = L.numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        want = expected(L, 6, 1e-2, 0.1)
    L.list.qsr_list_step(6, 1e-2)
    got = L.numpy()
    bad = [[300, 900], [7]]
    for i in range(2):
        assert np.isnan(got["p"][i][bad[i]]).all()
        ok = np.setdiff1d(np.arange(L.sizes[i]), bad[i])
        assert np.all(np.abs(got["p"][i][ok] - want[i][0][ok]) <= want[i][3][ok])
        assert np.isfinite(got["m"][i][ok]).all() and np.isfinite(got["v"][i][ok]).all()
        if states == "e4m3":
            assert np.isfinite(got["ms"][i]).all() and np.isfinite(got["vs"][i]).all()


def test_blocks_of_vanishing_magnitude_are_zeros():
    L = Lists([512], states="e4m3", n_old=0)
    L.g[0].fill_(1e-32)
    L.g[0][300] = 1e-3
    L.list.qsr_list_step(1, 1e-3)
    got = L.numpy()
    assert got["ms"][0][0] == 0 and (got["m"][0][:256] == 0).all() and got["ms"][0][1] > 0
    assert np.isfinite(got["p"][0]).all()


def test_gradients_allocated_anew():
    L = Lists([100, 5000], grad="bf16", weight_decay=0.1)
    fresh = [torch.randn(n, device=DEV).to(torch.bfloat16) for n in L.sizes]
    L.list.qsr_list_set_grads(fresh)
    L.g = fresh
    L.before = L.numpy()
    L.list.qsr_list_step(6, 1e-2)
    check_step(L, expected(L, 6, 1e-2, 0.1))


def test_transposed_parameters_share_their_order():
    p = torch.randn(48, 33, device=DEV).t()
    g, m, v = (torch.randn(48, 33, device=DEV).t() for _ in range(3))
    v.abs_()
    want = [x.double().cpu().numpy() for x in (p, g, m, v)]
    ws = torch.empty(B.qsr_list_workspace_bytes([p.numel()]), dtype=torch.uint8, device=DEV)
    lst = B.TensorList([p], [g], [m], [v], workspace=ws, stream=_stream())
    lst.qsr_list_step(3, 1e-2)
    th, g, m0, v0 = want
    m1, v1 = 0.9 * m0 + 0.1 * g, 0.999 * v0 + 0.001 * g * g
    th = th - 1e-2 / (1 - 0.9 ** 3) * m1 / (np.sqrt(v1 / (1 - 0.999 ** 3)) + 1e-8)
    assert np.allclose(p.double().cpu().numpy(), th, rtol=32 * U, atol=1e-6) and np.allclose(m.double().cpu().numpy(), m1, rtol=0, atol=8 * U * 4)


def test_python_refusals():
    p = torch.zeros(16, device=DEV)
    ws = torch.empty(4096, dtype=torch.uint8, device=DEV)
    f = lambda *s, **k: torch.zeros(*s, device=DEV, **k)      # noqa: E731
    ok = dict(workspace=ws, stream=_stream())
    with pytest.raises(ValueError):
        B.TensorList([p], [f(15)], [f(16)], [f(16)], **ok)
    with pytest.raises(ValueError):
        B.TensorList([p], [f(16, dtype=torch.float64)], [f(16)], [f(16)], **ok)
    with pytest.raises(ValueError):
        B.TensorList([p], [f(16)], [f(16, dtype=torch.bfloat16)], [f(16)], **ok)
    with pytest.raises(ValueError):
        B.TensorList([f(4, 4)], [f(4, 4).t()], [f(4, 4)], [f(4, 4)], **ok)          # other order in memory
    with pytest.raises(ValueError):
        B.TensorList([f(4, 8)[:, ::2]], [f(4, 8)[:, ::2]], [f(4, 8)[:, ::2]], [f(4, 8)[:, ::2]], **ok)
    with pytest.raises(ValueError):
        B.TensorList([p], [f(16)], [torch.zeros(16)], [f(16)], **ok)                 # on the CPU
    f8 = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        B.TensorList([p], [f(16)], [f(16).to(f8)], [f(16).to(f8)], **ok)            # no scales
    with pytest.raises(ValueError):
        B.TensorList([p], [f(16)], [f(16).to(f8)], [f(16).to(f8)], m_scale=[f(2)], v_scale=[f(1)], **ok)
    with pytest.raises(B.QsrError) as e:
        B.TensorList([p, p], [f(16), f(16)], [f(16), f(16)], [f(16), f(16)], **ok)   # the same tensor twice
    assert e.value.status == B.QSR_EINVAL
    with pytest.raises(B.QsrError) as e:
        B.TensorList([p, f(8)], [f(16), f(8)], [f(16), f(8)], [f(16), f(8)], workers=2, **ok)   # workers differ
    assert e.value.status == B.QSR_EINVAL
    with pytest.raises(B.QsrError) as e:
        B.TensorList([p], [f(16)], [f(16)], [f(16)], workspace=ws[:256], stream=_stream())
    assert e.value.status == B.QSR_ERANGE
    lst = B.TensorList([p], None, [f(16)], [f(16)], **ok)
    with pytest.raises(B.QsrError) as e:
        lst.qsr_list_step(1, 1e-3)
    assert e.value.status == B.QSR_ESTATE
    lst.qsr_list_set_grads([f(16)])
    with pytest.raises(B.QsrError) as e:
        lst.qsr_list_step(0, 1e-3)
    assert e.value.status == B.QSR_ERANGE
    for bad in (math.nan, math.inf):
        with pytest.raises(B.QsrError) as e:
            lst.qsr_list_step(1, bad)
        assert e.value.status == B.QSR_EINVAL
    assert lst.qsr_list_launch_count() == 0 and bool((p == 0).all())


@pytest.mark.parametrize("mode", ["keep", "average", "reset"])
@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("K,lead,types", [(1, 64, TYPES[0]), (2, 64, TYPES[1]), (3, 1, TYPES[3]), (5, 8, TYPES[2]), (16, 64, TYPES[4]), (33, 7, TYPES[0]),
                                          (70, 64, TYPES[3])])
def test_sync(K, lead, types, states, mode):
    param, grad, copy = types
    L = Lists([1, 257, 2048, 0, 3001], K=K, param=param, grad=grad, copy=copy, states=states, lead=lead, seed=K)
    L.list.qsr_list_sync(mode)
    got, b, n = L.numpy(), L.before, 5
    for j in range(n):
        if L.sizes[j] == 0:
            continue
        def per_worker(name):
            return np.stack([b[name][k * n + j] for k in range(K)])
        def same(name):
            return all(np.array_equal(got[name][k * n + j], got[name][j]) for k in range(K))
        th = per_worker("p")
        # K - 1 sums and a division in fp32, then the type's own rounding
        e = (K + 1) * U * np.abs(th).mean(0)
        mean = th.mean(0)
        assert same("p")
        assert np.all(np.abs(got["p"][j] - mean) <= e + HALF_ULP[param] * (np.abs(mean) + e) + TINY[param])
        if copy:
            assert same("c") and np.all(np.abs(got["c"][j] - mean) <= e + HALF_ULP[copy] * (np.abs(mean) + e) + TINY[copy])
        if mode == "keep":
            for name in ("m", "v", "ms", "vs"):
                assert b[name] is None or all(np.array_equal(got[name][k * n + j], b[name][k * n + j]) for k in range(K))
        elif mode == "reset":
            for name in ("m", "v", "ms", "vs"):
                assert b[name] is None or all((got[name][k * n + j] == 0).all() for k in range(K))
        elif states == "f32":
            for name in ("m", "v"):
                x = per_worker(name)
                assert same(name) and np.all(np.abs(got[name][j] - x.mean(0)) <= (K + 2) * U * np.abs(x).mean(0))
        else:
            m = np.stack([dequantise(b["m"][k * n + j], b["ms"][k * n + j]) for k in range(K)])
            u = np.stack([dequantise(b["v"][k * n + j], b["vs"][k * n + j]) for k in range(K)])
            for x, size, name, scale in ((m.mean(0), np.abs(m).mean(0), "m", "ms"), (np.sqrt((u * u).mean(0)), np.sqrt((u * u).mean(0)), "v", "vs")):
                assert same(name) and same(scale)
                e = (K + 4) * U * size
                amax = np.abs(blocks(x)).max(1)
                assert np.all(np.abs(got[scale][j] - amax / 448) <= blocks(e).max(1) / 448 + 2 * U * amax / 448)
                s = np.repeat(got[scale][j], 256)[:x.size]
                assert np.all(np.abs(got[name][j] * s - x) <= e + np.abs(x) * (2.0 ** -4 + 8 * U) + s * 2.0 ** -9)
    L.assert_guards()
    assert L.list.qsr_list_launch_count() == (2 if mode == "reset" else 1)


def test_sync_equals_the_slab_synchronization():
    """fp32 parameters: the same bits as qsr_sync gives on a [K, P] slab."""
    from paper_2310_14423_b200 import workloads as W
    w = W.tiny_workload(W.OPT_SGDM, K=5, P=4096)
    theta = torch.randn(5, 4096, device=DEV)
    rows = theta.clone()
    ctx = B.Context(B.make_config(w), theta, torch.zeros_like(theta), stream=_stream())
    ctx.qsr_sync(1)
    zeros = [torch.zeros(4096, device=DEV) for _ in range(10)]
    ws = torch.empty(B.qsr_list_workspace_bytes([4096] * 5, 5), dtype=torch.uint8, device=DEV)
    lst = B.TensorList(list(rows), None, zeros[:5], zeros[5:], workers=5, workspace=ws, stream=_stream())
    lst.qsr_list_sync("keep")
    assert torch.equal(theta, rows)


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_other_stream_and_graph_replay(states):
    """A list on a side stream; steps captured in a CUDA graph and replayed do what direct calls do."""
    direct = Lists([5000, 300], states=states, clip_norm=0.5)
    for _ in range(3):
        direct.list.qsr_list_step(6, 1e-3)
    want = direct.numpy()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        L = Lists([5000, 300], states=states, clip_norm=0.5)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            L.list.qsr_list_step(6, 1e-3)
        for _ in range(3):
            graph.replay()
        side.synchronize()
        got = L.numpy()
    for name in ("p", "m", "v"):
        assert all(np.array_equal(a, b) for a, b in zip(got[name], want[name]))


def test_many_chunks_and_offsets_beyond_32_bits():
    """One tensor of 2^31 + 777 elements: the last ones are stepped like a small tensor of the same values."""
    n, tail = (1 << 31) + 777, 3000
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    p, g = torch.zeros(n, device=DEV, dtype=bf), torch.zeros(n, device=DEV, dtype=bf)
    m, v = torch.zeros(n, device=DEV, dtype=torch.uint8).view(f8), torch.zeros(n, device=DEV, dtype=torch.uint8).view(f8)
    ms, vs = torch.zeros((n + 255) // 256, device=DEV), torch.zeros((n + 255) // 256, device=DEV)
    at = (n - tail) // 256 * 256
    p[at:], g[at:] = torch.randn(n - at, device=DEV).to(bf), torch.randn(n - at, device=DEV).to(bf)
    small = [x[at:].clone() for x in (p, g, m, v)] + [ms[at // 256:].clone(), vs[at // 256:].clone()]
    ws = torch.empty(B.qsr_list_workspace_bytes([n]), dtype=torch.uint8, device=DEV)
    big = B.TensorList([p], [g], [m], [v], m_scale=[ms], v_scale=[vs], workspace=ws, stream=_stream())
    big.qsr_list_step(1, 1e-2)
    ws2 = torch.empty(B.qsr_list_workspace_bytes([n - at]), dtype=torch.uint8, device=DEV)
    lst = B.TensorList(small[:1], small[1:2], small[2:3], small[3:4], m_scale=small[4:5], v_scale=small[5:], workspace=ws2, stream=_stream())
    lst.qsr_list_step(1, 1e-2)
    for a, b in ((p[at:], small[0]), (m[at:].view(torch.uint8), small[2].view(torch.uint8)), (vs[at // 256:], small[5])):
        assert torch.equal(a, b)
    assert bool((p[:1 << 20] == 0).all()) and float(ms[:at // 256].abs().max()) == 0.0


def test_tables_are_not_uploaded_during_a_capture():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        L = Lists([300])
        side.synchronize()
        ws = torch.empty_like(L.workspace)
        status = []
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for call in (lambda: L.list.qsr_list_set_grads(L.g),
                         lambda: B.TensorList([torch.zeros_like(x) for x in L.p], None, L.m, L.v, workspace=ws, stream=_stream())):
                try:
                    call()
                    status.append(0)
                except B.QsrError as e:
                    status.append(e.status)
            L.list.qsr_list_step(6, 1e-2)
        graph.replay()
        side.synchronize()
    assert status == [B.QSR_ESTATE, B.QSR_ESTATE]
    check_step(L, expected(L, 6, 1e-2, 0.0))


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("lead", [64, 1])
def test_gradients_whose_square_overflows(lead, grad, states):
    """Gradients of 3e19 (finite) and infinite ones, among ordinary neighbours and zeros, in whole blocks and ragged ends.  The
    formula in fp32: v and its root are infinite, so a finite gradient's update is 0; the root saturates at 448 in 8 bits."""
    n, lr, wd = 1300, 1e-2, 0.1
    big = {3: 3e19, 300: -3e19, 600: 3e19, 700: math.inf, 900: -math.inf, 1290: 3e19}
    L = Lists([n], grad=grad, states=states, lead=lead, weight_decay=wd, seed=11)
    L.wd[0] = 1.0
    L.list = B.TensorList(L.p, L.g, L.m, L.v, m_scale=L.ms, v_scale=L.vs, workspace=L.workspace, stream=_stream(), weight_decay=wd)
    codes = states == "e4m3"
    for lo, hi in ((296, 304), (512, 768)):                # zero neighbours: a lane's eight; a whole block, of gradients and states
        for x in (L.g, L.m, L.v):
            x[0][lo:hi].view(torch.uint8).zero_()
    for i, g in big.items():
        L.g[0][i] = g
    L.before = L.numpy()
    finite = [i for i in big if math.isfinite(big[i])]
    infinite = [i for i in big if not math.isfinite(big[i])]
    ordinary = np.setdiff1d(np.arange(n), list(big))
    with np.errstate(invalid="ignore", over="ignore"):
        want = expected(L, 6, lr, wd)
    L.list.qsr_list_step(6, lr)
    got = L.numpy()
    theta = L.before["p"][0]
    assert np.isnan(got["p"][0][infinite]).all()
    # the decay: factor and product rounded, then the difference
    assert np.all(np.abs(got["p"][0][finite] - theta[finite] * (1 - lr * wd)) <= 4 * U * np.abs(theta[finite]))
    assert np.all(np.abs(got["p"][0][ordinary] - want[0][0][ordinary]) <= want[0][3][ordinary] + TINY["f32"])
    m = np.asarray([0.1 * L.before["g"][0][i] for i in finite])
    if not codes:
        assert np.isposinf(got["v"][0][list(big)]).all() and np.isfinite(got["v"][0][ordinary]).all()
        assert np.all(np.abs(got["m"][0][finite] - m) <= 1e-6 * np.abs(m)) and np.isinf(got["m"][0][infinite]).all()
    else:
        block_of = lambda i: i // 256                      # noqa: E731
        assert np.isfinite(got["ms"][0]).all() and np.isfinite(got["vs"][0]).all()
        assert not np.isnan(got["m"][0]).any() and not np.isnan(got["v"][0]).any()
        assert np.all(np.abs(got["ms"][0][[block_of(i) for i in finite]] - np.abs(m) / 448) <= 1e-6 * np.abs(m) / 448)
        assert [got["m"][0][i] for i in finite] == [math.copysign(448.0, big[i]) for i in finite]
        # the block of 512..767 has no finite root above 0: it is stored as zeros
        assert [got["v"][0][i] for i in big] == [0.0 if block_of(i) == 2 else 448.0 for i in big]
        assert got["m"][0][900] == -448.0 and got["vs"][0][2] == 0 and (got["v"][0][512:768] == 0).all()
        amax = np.sqrt(blocks(np.where(np.isin(np.arange(n), list(big)), 0.0, want[0][2])).max(1))
        assert np.all(np.abs(got["vs"][0] - amax / 448) <= 16 * U * amax / 448)
    L.assert_guards()
    L.g[0].zero_()
    L.list.qsr_list_step(7, lr)
    after = L.numpy()
    assert np.isfinite(after["p"][0][ordinary]).all() and np.isnan(after["p"][0][infinite]).all()
    assert not codes or not (np.isnan(after["m"][0]).any() or np.isnan(after["v"][0]).any())


@pytest.mark.parametrize("lead", [64, 1])
def test_averaged_states_whose_sum_overflows(lead):
    """8-bit states: sums of m and of v beyond fp32 saturate at 448 in their element, or vanish with a block of zeros."""
    n, K = 1300, 3
    L = Lists([n], K=K, states="e4m3", lead=lead, seed=12)
    for k in range(K):
        for x, s, top in ((L.m[k], L.ms[k], 2.0e38), (L.v[k], L.vs[k], 1.7e19)):
            byte = x.view(torch.uint8)
            byte[:256] = torch.arange(256, device=DEV) % 16 + 0x30          # 0.5 .. 1.9
            byte[512:768] = 0
            byte[1024:] = 0
            for i in (5, 600, 1290):
                byte[i] = 0x7e + 0x80 * (x is L.m[k] and i != 600)           # 448, or -448
                s[i // 256] = top / 448
    before = L.numpy()
    L.list.qsr_list_sync("average")
    got = L.numpy()
    for name, scale, sign in (("m", "ms", -1.0), ("v", "vs", 1.0)):
        ordinary = [np.setdiff1d(np.arange(256), [5]), np.arange(256, 512), np.arange(768, 1024)]
        for k in range(K):
            assert np.isfinite(got[scale][k]).all() and not np.isnan(got[name][k]).any()
            assert got[name][k][5] == sign * 448.0
            for block in (2, 5):
                assert got[scale][k][block] == 0 and (got[name][k][block * 256:(block + 1) * 256] == 0).all()
            assert np.array_equal(got[name][k], got[name][0]) and np.array_equal(got[scale][k], got[scale][0])
        for span in ordinary:
            x = np.stack([dequantise(before[name][k], before[scale][k])[span] for k in range(K)])
            e = (K + 4) * U * np.abs(x).max(0)
            x = x.mean(0) if name == "m" else np.sqrt((x * x).mean(0))
            s = got[scale][0][span[0] // 256]
            assert abs(s - np.abs(x).max() / 448) <= e.max() / 448 + 2 * U * np.abs(x).max() / 448
            assert np.all(np.abs(got[name][0][span] * s - x) <= e + np.abs(x) * (2.0 ** -4 + 8 * U) + s * 2.0 ** -9)
    L.assert_guards()


def test_gradient_table_in_page_locked_memory():
    """The table is read during the call only, whatever memory it lies in: it is overwritten while the stream is still busy."""
    L = Lists([100, 5000], grad="bf16", weight_decay=0.1)
    fresh = [torch.randn(n, device=DEV).to(torch.bfloat16) for n in L.sizes]
    others = [torch.zeros_like(g) for g in fresh]
    table = torch.tensor([g.data_ptr() for g in fresh], dtype=torch.int64).pin_memory()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                         # about 50 ms
    assert B.lib().qsr_list_set_grads(L.list._h, table.data_ptr()) == B.QSR_OK
    table.copy_(torch.tensor([g.data_ptr() for g in others], dtype=torch.int64))
    L.list.qsr_list_step(6, 1e-2)
    L.g = fresh
    L.before["g"] = [g.double().cpu().numpy() for g in fresh]
    check_step(L, expected(L, 6, 1e-2, 0.1))


def test_no_upload_while_a_blocking_stream_is_captured():
    """A list on the legacy default stream while another, blocking stream is being captured: refused, and the capture goes on."""
    L = Lists([300])
    lst = B.TensorList(L.p, L.g, L.m, L.v, workspace=L.workspace)           # stream 0
    torch.cuda.synchronize()
    raw = C.c_void_p()
    assert int(torch.cuda.cudart().cudaStreamCreate(C.addressof(raw))) == 0
    blocking = torch.cuda.ExternalStream(raw.value)
    x, other = torch.zeros(8, device=DEV), torch.empty_like(L.workspace)
    spare = [torch.zeros_like(t) for t in L.p]
    status = []
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=blocking):
        x.add_(1.0)
        for call in (lambda: lst.qsr_list_set_grads(L.g), lambda: B.TensorList(spare, None, L.m, L.v, workspace=other)):
            try:
                call()
                status.append(0)
            except B.QsrError as e:
                status.append(e.status)
        x.add_(1.0)
    x.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert status == [B.QSR_ESTATE, B.QSR_ESTATE] and bool((x == 2.0).all())
    lst.qsr_list_step(6, 1e-2)
    torch.cuda.synchronize()
    check_step(L, expected(L, 6, 1e-2, 0.0))


@pytest.mark.parametrize("again", [False, True])
def test_replaced_gradients_stay_until_the_list_has_read_them(again):
    """Gradients of another stream than the list's, dropped by everybody when they are replaced: their memory is not given out
    again while the list's stream has yet to read them."""
    L = Lists([100, 5000], weight_decay=0.1)
    side = torch.cuda.Stream()
    lst = B.TensorList(L.p, L.g, L.m, L.v, wd_scale=L.wd, workspace=L.workspace, stream=side.cuda_stream, weight_decay=0.1)
    values = [torch.randn(n, device=DEV) for n in L.sizes]
    torch.cuda.synchronize()
    if again:                                              # gradients that the list was given by the call, not when it was made
        lst.qsr_list_set_grads([x.clone() for x in values])
    else:
        grads = [x.clone() for x in values]
        lst = B.TensorList(L.p, grads, L.m, L.v, wd_scale=L.wd, workspace=L.workspace, stream=side.cuda_stream, weight_decay=0.1)
        grads.clear()                                      # the list keeps the tensors, not the caller's container
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)                     # about 50 ms
    lst.qsr_list_step(6, 1e-2)
    # memory of the current stream
    lst.qsr_list_set_grads([torch.zeros(n, device=DEV) for n in L.sizes])
    taken = [torch.full((n,), math.nan, device=DEV) for n in L.sizes for _ in range(4)]
    torch.cuda.synchronize()
    L.before["g"] = [x.double().cpu().numpy() for x in values]
    check_step(L, expected(L, 6, 1e-2, 0.1))
    assert all(bool(x.isnan().all()) for x in taken)


LARGE = [1_900_003, 8191, 8192, 8193, 600_000, 33, 0, 24_577]      # beyond 2,424,832 elements a warp has several blocks


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("lead,types", [(64, TYPES[1]), (1, TYPES[3]), (3, TYPES[0]), (8, TYPES[4])])
def test_step_of_a_large_list(lead, types, states):
    param, grad, copy = types
    L = Lists(LARGE, param=param, grad=grad, copy=copy, states=states, lead=lead, weight_decay=0.1, seed=20 + lead)
    L.list.qsr_list_step(6, 1e-2)
    check_step(L, expected(L, 6, 1e-2, 0.1))


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("lead", [64, 5])
def test_clipping_of_a_large_list(lead, states):
    norms = torch.zeros(2, device=DEV)
    L = Lists([1_300_001, 8192, 24_577, 7], K=2, grad="bf16", copy="bf16", states=states, lead=lead, clip_norm=0.5, grad_norm=norms, weight_decay=0.05,
              seed=30)
    L.list.qsr_list_step(4, 1e-3)
    check_step(L, expected(L, 4, 1e-3, 0.05, clip=0.5))
    want = [math.sqrt(sum(float((g * g).sum()) for g in L.before["g"][4 * k:4 * k + 4])) for k in range(2)]
    assert np.allclose(norms.cpu().numpy(), want, rtol=64 * U, atol=0)


@pytest.mark.parametrize("mode", ["keep", "average", "reset"])
@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("lead,types", [(64, TYPES[1]), (1, TYPES[3])])
def test_sync_of_a_large_list_equals_a_list_per_tensor(lead, types, states, mode):
    """The same bits, whatever the chunks: workers are added in ascending order.  Lists of one tensor here are small ones."""
    param, grad, copy = types
    sizes, K = [750_001, 8193, 100_000, 33], 3
    one, many = (Lists(sizes, K=K, param=param, grad=grad, copy=copy, states=states, lead=lead, seed=40) for _ in range(2))
    one.list.qsr_list_sync(mode)
    for j in range(len(sizes)):
        pick = lambda xs: None if xs is None else xs[j::len(sizes)]      # noqa: E731
        ws = torch.empty(B.qsr_list_workspace_bytes([sizes[j]] * K, K), dtype=torch.uint8, device=DEV)
        lst = B.TensorList(pick(many.p), None, pick(many.m), pick(many.v), m_scale=pick(many.ms), v_scale=pick(many.vs), copies=pick(many.c), workers=K,
                           workspace=ws, stream=_stream())
        lst.qsr_list_sync(mode)
    a, b = one.numpy(), many.numpy()
    for name in ("p", "c", "m", "v", "ms", "vs"):
        assert a[name] is None or all(np.array_equal(x, y) for x, y in zip(a[name], b[name])), name
    mean = np.mean([one.before["p"][k * len(sizes)] for k in range(K)], 0)
    e = (K + 1) * U * np.abs(mean).max() * 4
    assert np.all(np.abs(a["p"][0] - mean) <= e + HALF_ULP[param] * (np.abs(mean) + e) + TINY[param])
    one.assert_guards()
    many.assert_guards()


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("lead", [64, 3])
def test_several_types_in_one_list(lead, states):
    """fp32 vectors beside bf16 and fp16 matrices, with gradients and copies of their own types, in one step and one mean."""
    K = 2
    groups = [Lists(sizes, K=K, param=t[0], grad=t[1], copy=t[2], states=states, lead=lead, seed=50 + i)
              for i, (sizes, t) in enumerate((([7, 300, 2049], TYPES[0]), ([4100, 33], TYPES[3]), ([8200, 1], TYPES[1]), ([513], TYPES[4]), ([777], TYPES[5])))]

    def merged(name):
        """Worker 0's tensors of all groups, then worker 1's."""
        out = []
        for k in range(K):
            for L in groups:
                n, xs = len(L.sizes), getattr(L, name)
                out += [None] * n if xs is None else xs[k * n:(k + 1) * n]
        return out

    codes = states == "e4m3"
    every = [x.numel() for x in merged("p")]
    ws = torch.empty(B.qsr_list_workspace_bytes(every, K), dtype=torch.uint8, device=DEV)
    lst = B.TensorList(merged("p"), merged("g"), merged("m"), merged("v"), m_scale=merged("ms") if codes else None,
                       v_scale=merged("vs") if codes else None, copies=merged("c"), wd_scale=merged("wd"), workers=K, workspace=ws, stream=_stream(),
                       weight_decay=0.1)
    lst.qsr_list_step(6, 1e-2)
    for L in groups:
        check_step(L, expected(L, 6, 1e-2, 0.1))
    before = [L.numpy() for L in groups]
    lst.qsr_list_sync("average")
    for L, b in zip(groups, before):
        got, n = L.numpy(), len(L.sizes)
        for j in range(n):
            th = np.stack([b["p"][k * n + j] for k in range(K)])
            e = (K + 1) * U * np.abs(th).mean(0)
            param = L.types[0]
            for k in range(K):
                assert np.all(np.abs(got["p"][k * n + j] - th.mean(0)) <= e + HALF_ULP[param] * (np.abs(th.mean(0)) + e) + TINY[param])
                assert all(got[x] is None or np.array_equal(got[x][k * n + j], got[x][j]) for x in ("p", "c", "m", "v", "ms", "vs"))
        L.assert_guards()
