"""What ks_quantize_e4m3, ks_matmul_e4m3 and ks_sample refuse, without a GPU: arguments are checked before the context is used,
so a block of zeros stands in for one, and no pointer is followed."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2609_35587_b200 import binding as ks

CTX = ctypes.create_string_buffer(4096)
P = 1 << 20  # an address that is never used
OVER = (1 << 31) - 1023  # rows or columns, one too many


def call(fn, *args):
    return int(fn(ctypes.cast(CTX, ctypes.c_void_p), *args))


QUANT = dict(x=P, x_type=ks.KS_F32, rows=4, cols=200, ldx=200, block_rows=1, scale_type=ks.KS_SCALE_E8M0, q=P, ldq=208, scale=P)


def quantize(**kw):
    a = dict(QUANT, **kw)
    return call(ks._lib.ks_quantize_e4m3, a["x"], a["x_type"], a["rows"], a["cols"], a["ldx"], a["block_rows"], a["scale_type"],
                a["q"], a["ldq"], a["scale"], None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(q=None), dict(scale=None), dict(x_type=3), dict(x_type=-1), dict(rows=-1), dict(cols=-1), dict(ldx=199),
    dict(ldq=199), dict(ldq=200), dict(q=P + 8), dict(x=P + 2), dict(block_rows=64), dict(block_rows=0), dict(scale_type=2),
    dict(scale=P + 2, scale_type=ks.KS_SCALE_F32), dict(rows=1 << 31), dict(cols=1 << 31, ldx=1 << 31, ldq=1 << 31),
    dict(rows=OVER), dict(cols=OVER, ldx=1 << 31, ldq=1 << 31)])
def test_quantize(bad):
    assert quantize(**bad) == ks.KS_ERR_INVALID_ARG


def test_nothing_to_do():
    assert quantize(rows=0, x=None, q=None, scale=None) == ks.KS_OK
    assert quantize(cols=0, ldx=0, x=None, q=None, scale=None) == ks.KS_OK
    assert matmul(m=0, a=None, d=None) == ks.KS_OK
    assert matmul(n=0, b=None, d=None) == ks.KS_OK
    assert sample(P=0, scores=None, u=None, idx=None) == ks.KS_OK


MATMUL = dict(a=P, lda=208, sa=P, b=P, ldb=208, sb=P, scale_type=ks.KS_SCALE_F32, m=4, n=8, k=200, bias=None, relu=0, d=P,
              ldd=8, d_type=ks.KS_F32, sd=None)


def matmul(**kw):
    a = dict(MATMUL, **kw)
    return call(ks._lib.ks_matmul_e4m3, a["a"], a["lda"], a["sa"], a["b"], a["ldb"], a["sb"], a["scale_type"], a["m"], a["n"], a["k"],
                a["bias"], a["relu"], a["d"], a["ldd"], a["d_type"], a["sd"], None)


@pytest.mark.parametrize("bad", [
    dict(a=None), dict(b=None), dict(sa=None), dict(sb=None), dict(d=None), dict(lda=199), dict(lda=200), dict(ldb=192), dict(ldb=216),
    dict(a=P + 8), dict(b=P + 4), dict(sa=P + 1), dict(sb=P + 2), dict(bias=P + 2), dict(d=P + 2), dict(ldd=7), dict(m=-1), dict(n=-1),
    dict(k=-1), dict(m=1 << 31), dict(d_type=4), dict(d_type=-1), dict(scale_type=7), dict(sd=P), dict(d_type=ks.KS_E4M3),
    dict(d_type=ks.KS_E4M3, sd=P, ldd=8), dict(d_type=ks.KS_E4M3, sd=P, ldd=16, d=P + 1), dict(d_type=ks.KS_E4M3, sd=P + 2, ldd=16),
    dict(m=OVER), dict(n=OVER, ldd=1 << 31), dict(k=OVER, lda=1 << 31, ldb=1 << 31)])
def test_matmul(bad):
    assert matmul(**bad) == ks.KS_ERR_INVALID_ARG


SAMPLE = dict(scores=P, score_type=ks.KS_F32, P=3, c=10, ld=10, seg=None, t=1.0, top_k=0, top_p=1.0, min_p=0.0, params=None, u=P,
              draws=1, idx=P, logp=None, none=False)


def sample(**kw):
    a = dict(SAMPLE, **kw)
    one = ks._Sampling(a["t"], a["top_k"], a["top_p"], a["min_p"])
    return call(ks._lib.ks_sample, a["scores"], a["score_type"], a["P"], a["c"], a["ld"], a["seg"],
                None if a["none"] else ctypes.byref(one), a["params"], a["u"], a["draws"], a["idx"], a["logp"], None)


@pytest.mark.parametrize("bad", [
    dict(scores=None), dict(u=None), dict(idx=None), dict(P=-1), dict(c=-1), dict(ld=9), dict(c=1 << 31, ld=1 << 31), dict(seg=P, c=-1), dict(draws=0), dict(draws=33), dict(score_type=3),
    dict(score_type=-1), dict(scores=P + 2), dict(params=P + 2), dict(seg=P + 4), dict(none=True), dict(t=-1.0), dict(t=float("nan")),
    dict(t=float("inf")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.5), dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.1),
    dict(min_p=float("nan")), dict(c=OVER, ld=1 << 31), dict(u=P + 2), dict(idx=P + 1), dict(logp=P + 2)])
def test_sample(bad):
    assert sample(**bad) == ks.KS_ERR_INVALID_ARG


def test_no_context():
    one = ks._Sampling(1.0, 0, 1.0, 0.0)
    assert ks._lib.ks_quantize_e4m3(None, P, 0, 1, 1, 1, 1, 0, P, 16, P, None) == ks.KS_ERR_INVALID_ARG
    assert ks._lib.ks_matmul_e4m3(None, P, 16, P, P, 16, P, 0, 1, 1, 16, None, 0, P, 1, 0, None, None) == ks.KS_ERR_INVALID_ARG
    assert ks._lib.ks_sample(None, P, 0, 1, 1, 1, None, ctypes.byref(one), None, P, 1, P, None, None) == ks.KS_ERR_INVALID_ARG


def test_sampling_records_are_the_c_struct():
    assert ks.SAMPLING_DT.itemsize == ctypes.sizeof(ks._Sampling) == 16
    r = np.zeros(1, ks.SAMPLING_DT)
    r["temperature"], r["top_k"], r["top_p"], r["min_p"] = 0.5, 7, 0.25, 0.125
    s = ks._Sampling.from_buffer_copy(r.tobytes())
    assert (s.temperature, s.top_k, s.top_p, s.min_p) == (0.5, 7, 0.25, 0.125)


def test_model_in_eight_bits():
    widths = np.array([64, 64, 1], np.int32)
    one = np.ones(64 * 64, np.float32)
    w = (ctypes.c_void_p * 2)(P, P)
    out = ctypes.c_void_p()

    def create(n_layers, widths, sigma=one):
        return call(ks._lib.ks_model_create_mlp_e4m3, n_layers, widths.ctypes.data, ctypes.cast(w, ctypes.c_void_p),
                    ctypes.cast(w, ctypes.c_void_p), one.ctypes.data, sigma.ctypes.data, ctypes.byref(out))
    assert create(1, np.array([64, 1], np.int32)) == ks.KS_ERR_INVALID_ARG  # a linear scorer has no layer to quantise
    assert create(2, np.array([64, 100, 1], np.int32)) == ks.KS_ERR_INVALID_ARG
    assert create(2, np.array([72, 64, 1], np.int32)) == ks.KS_ERR_INVALID_ARG
    assert create(7, widths) == ks.KS_ERR_INVALID_ARG
    assert create(2, widths, np.zeros(64, np.float32)) == ks.KS_ERR_INVALID_ARG
    assert out.value is None


def test_binding_wants_the_context_device():
    """Tensors in host memory or on another GPU are not handed over."""
    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1
    there = torch.zeros(2, 4).as_subclass(Elsewhere)
    for fn in (ks._rows, ks._flat):
        for t in (torch.zeros(2, 4), there):
            with pytest.raises(ValueError):
                fn(t, 0)
        assert fn(there, 1)


class Recorded:
    """In the place of the library: what it is called with."""
    call = None

    def __getattr__(self, name):
        def fn(*args):
            self.call = (name, args)
            return ks.KS_OK
        return fn


class Handle:
    class device:
        index = -1  # (of tensors in host memory)
    _h = None


@pytest.fixture
def recorded(monkeypatch):
    lib = Recorded()
    monkeypatch.setattr(ks, "_lib", lib)
    monkeypatch.setattr(ks, "_raw_stream", lambda device: 0)
    return lib


@pytest.mark.parametrize("v", [1 << 31, (1 << 32) + 1, (1 << 32) + 128, -(1 << 31) - 1, -(1 << 32) + 1])
def test_numbers_that_32_bits_do_not_hold(recorded, v):
    """They are refused: wrapped, block_rows would write more scales than the binding made room for, and top_k would be another."""
    x, u = torch.zeros(4, 200), torch.zeros(4, 2)
    with pytest.raises(ValueError):
        ks.Context.quantize_e4m3(Handle, x, block_rows=v)
    with pytest.raises(ValueError):
        ks.Context.sample(Handle, x, u, top_k=v)
    assert recorded.call is None


def test_whole_numbers_of_other_types(recorded):
    x, u = torch.zeros(4, 200), torch.zeros(4, 2)
    ks.Context.quantize_e4m3(Handle, x, block_rows=np.int64(128))
    assert recorded.call[1][6] == 128
    ks.Context.sample(Handle, x, u, top_k=np.int64(7))
    assert recorded.call[1][7]._obj.top_k == 7
    q, s = torch.zeros(4, 128).to(torch.float8_e4m3fn), torch.zeros(4, 1)
    for relu, want in ((1 << 32, 1), (True, 1), (0, 0)):
        ks.Context.matmul_e4m3(Handle, q, s, q, s[:1], relu=relu)
        assert recorded.call[1][12] == want


def test_dependent_kernels_load_what_the_one_in_front_wrote():
    """The operators' kernels begin while the one in front still writes: no load through the read-only path, which may be moved or kept."""
    csrc = os.path.join(os.path.dirname(ks.__file__), "csrc")
    dependents = [f for f in sorted(os.listdir(csrc)) if "  wait_for_last();" in open(os.path.join(csrc, f)).read()]
    assert dependents == ["ks_matmul8.cu", "ks_quant.cu", "ks_sample.cu"]
    for f in dependents + ["ks_e4m3.cuh"]:
        code = re.sub(r"//.*", "", open(os.path.join(csrc, f)).read())
        assert not re.search(r"__ldg|ld\.global\.nc|__restrict__", code), f


@pytest.mark.parametrize("shape", [(1, (1 << 32) + 1), ((1 << 32) + 3, 1), (1 << 31, 2)])
def test_more_draws_than_32_bits_count(recorded, shape):
    u = torch.zeros(1).expand(shape)  # (one number's memory)
    with pytest.raises(ValueError, match="sizes of u"):
        ks.Context.sample(Handle, torch.zeros(1, 5).expand(shape[0], 5), u)
    assert recorded.call is None
