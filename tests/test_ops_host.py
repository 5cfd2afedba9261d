"""Refusals and host arithmetic of the operators on microscaled rows, rotary positions and key intervals: no GPU.
Every refused call returns before anything is enqueued, so made-up device addresses are never read."""
import ctypes as C
import math
import os

import numpy as np
import pytest

import ops_reference as R

P = pytest.importorskip("paper_2609_29505_amd")
A, B, D, E, F = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000  # aligned addresses


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(P.lib_path):
        pytest.skip("libsgd.so not built")
    return P.lib()


ARG, SHAPE, DTYPE = -1, -2, -3


def refused(rc, code, L):
    assert rc == code, (rc, L.sgd_last_error())
    assert L.sgd_last_error()


def test_mx_bytes(L):
    c, s = C.c_size_t(), C.c_size_t()
    assert L.sgd_op_mx_bytes(0, 5, 288, C.byref(c), C.byref(s)) == 0 and (c.value, s.value) == (5 * 288, 2 * 5 * 8)
    assert L.sgd_op_mx_bytes(1, 5, 288, C.byref(c), C.byref(s)) == 0 and (c.value, s.value) == (5 * 144, 2 * 5 * 8)
    refused(L.sgd_op_mx_bytes(2, 5, 288, C.byref(c), C.byref(s)), DTYPE, L)
    refused(L.sgd_op_mx_bytes(0, 0, 288, C.byref(c), C.byref(s)), SHAPE, L)
    refused(L.sgd_op_mx_bytes(0, 5, 48, C.byref(c), C.byref(s)), SHAPE, L)
    refused(L.sgd_op_mx_bytes(0, 5, 64, None, C.byref(s)), ARG, L)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), ARG), (dict(codes=None), ARG), (dict(scales=None), ARG), (dict(fmt=2), DTYPE), (dict(dtype=2), DTYPE),
    (dict(rows=0), SHAPE), (dict(K=40), SHAPE), (dict(K=0), SHAPE), (dict(rows=1 << 20, K=1 << 14, ld=1 << 14), SHAPE), (dict(ld=32), ARG),
    (dict(ld=68), ARG), (dict(x=A + 8), ARG), (dict(codes=B + 8), ARG), (dict(scales=D + 4), ARG)])
def test_quantize_refuses(L, change, code):
    a = dict(fmt=0, dtype=1, x=A, ld=64, rows=3, K=64, codes=B, scales=D)
    a.update(change)
    refused(L.sgd_op_mx_quantize(a["fmt"], a["dtype"], a["x"], a["ld"], a["rows"], a["K"], a["codes"], a["scales"], None), code, L)
    refused(L.sgd_op_mx_dequantize(a["fmt"], a["codes"], a["scales"], a["rows"], a["K"], a["dtype"], a["x"], a["ld"], None), code, L)


@pytest.mark.parametrize("change,code", [
    (dict(a=None), ARG), (dict(sw=None), ARG), (dict(out=None), ARG), (dict(fmt=3), DTYPE), (dict(odt=2), DTYPE), (dict(act=4), ARG),
    (dict(tile=9), ARG), (dict(tile=-1), ARG), (dict(odt=0, act=1), DTYPE), (dict(odt=0, gated=1), DTYPE), (dict(M=0), SHAPE), (dict(N=6), SHAPE),
    (dict(K=16), SHAPE), (dict(K=80), SHAPE), (dict(gated=1, N=36, ldo=36), SHAPE), (dict(ldo=60), ARG), (dict(ldo=66), ARG), (dict(out=E + 4), ARG),
    (dict(odt=0, out=E + 8), ARG), (dict(bias=F + 4), ARG), (dict(a=A + 8), ARG), (dict(w=B + 8), ARG), (dict(sa=D + 4), ARG),
    (dict(tile=8, M=17), SHAPE), (dict(tile=1, gated=1, N=64), SHAPE), (dict(N=1 << 22, ldo=1 << 22, K=1 << 12), SHAPE)])
def test_linear_refuses(L, change, code):
    a = dict(fmt=0, a=A, sa=D, w=B, sw=D, bias=None, odt=1, out=E, ldo=64, M=4, N=64, K=64, act=0, gated=0, tile=0)
    a.update(change)
    refused(L.sgd_op_linear_mx(*[a[k] for k in ("fmt", "a", "sa", "w", "sw", "bias", "odt", "out", "ldo", "M", "N", "K", "act", "gated", "tile")],
                               None), code, L)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), ARG), (dict(xo=None), ARG), (dict(w=None), ARG), (dict(codes=None), ARG), (dict(fmt=-1), DTYPE), (dict(xdt=5), DTYPE),
    (dict(adt=5), DTYPE), (dict(M=0), SHAPE), (dict(d=16), SHAPE), (dict(d=8224), SHAPE), (dict(d=100), SHAPE), (dict(eps=-1.0), ARG),
    (dict(eps=math.nan), ARG), (dict(x=A + 8), ARG), (dict(add=A + 4), ARG), (dict(w=B + 4), ARG), (dict(scales=D + 1), ARG)])
def test_norm_refuses(L, change, code):
    a = dict(fmt=0, xdt=0, x=A, adt=1, add=E, xo=A, w=B, eps=1e-5, M=3, d=64, codes=F, scales=D)
    a.update(change)
    refused(L.sgd_op_norm_add_mx(*[a[k] for k in ("fmt", "xdt", "x", "adt", "add", "xo", "w", "eps", "M", "d", "codes", "scales")], None), code, L)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), ARG), (dict(turns=None), ARG), (dict(dt=2), DTYPE), (dict(T=0), SHAPE), (dict(H=0), SHAPE), (dict(H=70000), SHAPE),
    (dict(dh=258), SHAPE), (dict(rot=7), SHAPE), (dict(rot=66), SHAPE), (dict(rot=0), SHAPE), (dict(x=A + 1), ARG), (dict(turns=B + 4), ARG),
    (dict(pos=D + 2), ARG), (dict(ot=0), ARG), (dict(oh=0), ARG), (dict(out=A, ot=512), ARG)])
def test_rotary_refuses(L, change, code):
    a = dict(dt=1, x=A, xt=256, xh=64, out=E, ot=256, oh=64, T=3, H=4, dh=64, rot=64, inter=0, pos=D, turns=B, mag=1.0, inv=0)
    a.update(change)
    refused(L.sgd_op_rotary(*[a[k] for k in ("dt", "x", "xt", "xh", "out", "ot", "oh", "T", "H", "dh", "rot", "inter", "pos", "turns", "mag", "inv")],
                            None), code, L)


def _call(**kw):
    from paper_2609_29505_amd.binding import sgd_range_attention
    d = dict(q=A, k=B, v=D, o=E, q_stride=(512, 256, 64), k_stride=(512, 256, 64), v_stride=(512, 256, 64), o_stride=(512, 256, 64), ranges=F,
             pos=None, slopes=None, B=1, H=4, Hk=4, dh=64, nq=2, nk=2, scale=0.0, cap=0.0)
    d.update(kw)
    strides = (*d["q_stride"], *d["k_stride"], *d["v_stride"], *d["o_stride"])
    return sgd_range_attention(d["q"], d["k"], d["v"], d["o"], strides, d["ranges"], d["pos"], d["slopes"], d["B"], d["H"], d["Hk"], d["dh"], d["nq"], d["nk"], d["scale"], d["cap"])


@pytest.mark.parametrize("dt,change,code", [
    (2, {}, DTYPE), (1, dict(B=0), SHAPE), (1, dict(Hk=3), SHAPE), (1, dict(Hk=0), SHAPE), (1, dict(dh=136), SHAPE), (1, dict(dh=12), SHAPE),
    (1, dict(nq=0), SHAPE), (1, dict(nk=0), SHAPE), (1, dict(B=20000), SHAPE), (1, dict(q_stride=(512, 252, 64)), ARG),
    (1, dict(k_stride=(512, 256, 60)), ARG), (1, dict(k_stride=(512, 56, 64)), ARG), (1, dict(v_stride=(512, 1 << 24, 64)), ARG),
    (1, dict(v_stride=(512, 0, 64)), ARG), (1, dict(o_stride=(512, 254, 64)), ARG), (1, dict(scale=-1.0), ARG), (1, dict(cap=-1.0), ARG),
    (1, dict(cap=math.inf), ARG), (1, dict(scale=math.nan), ARG), (1, dict(q=None), ARG), (1, dict(ranges=None), ARG), (1, dict(k=B + 8), ARG),
    (1, dict(o=E + 4), ARG), (0, dict(o=E + 8), ARG)])
def test_attention_refuses(L, dt, change, code):
    refused(L.sgd_op_attention_ranges(dt, C.byref(_call(**change)), None, 0, None), code, L)


def test_attention_workspace(L):
    """Long caches with few query rows need one; a short call does not, and a missing or small one is refused."""
    n = C.c_size_t()
    assert L.sgd_op_attention_ranges_bytes(1, C.byref(_call()), C.byref(n)) == 0 and n.value == 0
    long = _call(nq=1, nk=1 << 16, k_stride=(1 << 24, 256, 64), v_stride=(1 << 24, 256, 64))
    assert L.sgd_op_attention_ranges_bytes(1, C.byref(long), C.byref(n)) == 0 and n.value > 0
    refused(L.sgd_op_attention_ranges(1, C.byref(long), None, 0, None), ARG, L)
    refused(L.sgd_op_attention_ranges(1, C.byref(long), A, n.value - 1, None), ARG, L)
    refused(L.sgd_op_attention_ranges(1, C.byref(long), A + 4, n.value, None), ARG, L)
    refused(L.sgd_op_attention_ranges_bytes(1, None, C.byref(n)), ARG, L)


@pytest.mark.parametrize("rot", [4, 64, 128])
def test_rope_turns(L, rot):
    i = np.arange(rot // 2)
    plain = 10000.0 ** (-2 * i / rot) / (2 * np.pi)
    t, m = P.rope_turns(rot)
    assert np.allclose(t, plain, rtol=1e-14) and m == 1.0
    t, m = P.rope_turns(rot, scaling="linear", factor=8)
    assert np.allclose(t, plain / 8, rtol=1e-14) and m == 1.0
    t, m = P.rope_turns(rot, scaling="base", factor=8)
    # the fastest pair is kept, the slowest one divided by the factor
    assert np.isclose(t[0], plain[0], rtol=1e-14) and np.isclose(t[-1], plain[-1] / 8, rtol=1e-12) and m == 1.0
    t, m = P.rope_turns(rot, scaling="parts", factor=8, context=4096, low=1, high=32)
    turns = plain * 4096
    assert np.allclose(t[turns >= 32], plain[turns >= 32], rtol=1e-14)
    assert np.allclose(t[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    g = (turns[mid] - 1) / 31
    assert np.allclose(t[mid], plain[mid] * (g + (1 - g) / 8), rtol=1e-13)
    assert np.isclose(m, 0.1 * math.log(8) + 1, rtol=1e-15)


@pytest.mark.parametrize("kw", [dict(rot=3), dict(rot=0), dict(rot=64, base=0.0), dict(rot=64, scaling="linear", factor=0.5),
                                dict(rot=2, scaling="base", factor=2.0), dict(rot=64, scaling="parts", factor=2.0, context=0.0),
                                dict(rot=64, scaling="parts", factor=2.0, context=4096.0, low=4.0, high=4.0),
                                dict(rot=64, scaling="linear", factor=math.nan)])
def test_rope_turns_refuses(L, kw):
    with pytest.raises(P.SgdError):
        P.rope_turns(**kw)


def test_reference_quantiser():
    """The tests' own quantiser on values worked out by hand."""
    x = np.zeros((1, 32))
    x[0, :8] = [6.0, -0.25, 0.75, 1.25, 2.5, 5.0, 7.9, -3.5]
    c, s = R.quantize(x, "fp4")
    assert s[0, 0] == 127  # max 7.9 in [4, 8): scale 2^(2 - 2)
    assert list(c[0, :8]) == [7, 8, 2, 2, 4, 6, 7, 14]
    x[0, :4] = [448.0, 449.0, 511.0, 2.0 ** -10]
    c, s = R.quantize(x, "fp8")
    assert s[0, 0] == 127 and list(c[0, :4]) == [126, 126, 126, 0]  # 2^-10: half the smallest, ties to even
    x[0, 0] = np.inf
    c, s = R.quantize(x, "fp8")
    assert s[0, 0] == 255 and not c.any()


def test_launches_past_the_grid_are_refused(L):
    """A launch has at most 2^32 threads; tensors that would need more are refused before any."""
    refused(L.sgd_op_norm_add_mx(0, 1, A, 1, None, None, B, 1e-5, 1 << 24, 32, F, D, None), SHAPE, L)
    refused(L.sgd_op_rotary(1, A, 64, 64, E, 64, 64, 1 << 24, 1, 64, 64, 0, None, B, 1.0, 0, None), SHAPE, L)
    refused(L.sgd_op_linear_mx(1, A, D, B, D, None, 1, E, 1 << 27, 16, 1 << 27, 32, 0, 0, 0, None), SHAPE, L)  # 2^23 workgroups of 512
    refused(L.sgd_op_linear_mx(1, A, D, B, D, None, 1, E, 1 << 20, 1 << 24, 1 << 20, 32, 0, 0, 0, None), SHAPE, L)
    refused(L.sgd_op_attention_ranges(1, C.byref(_call(B=1 << 13, nq=1 << 18)), None, 0, None), SHAPE, L)


@pytest.mark.parametrize("dt,change", [
    (1, dict(o_stride=(512, 0, 64))), (1, dict(o_stride=(512, 256, 0))), (1, dict(B=2, o_stride=(0, 256, 64))), (1, dict(cap=1025.0)),
    (0, dict(cap=1e-38, scale=100.0))])
def test_attention_refuses_outputs_and_caps(L, dt, change):
    refused(L.sgd_op_attention_ranges(dt, C.byref(_call(**change)), None, 0, None), ARG, L)


class _Buffer:
    """Stands for a device tensor of a call that reaches no GPU."""

    def __init__(self, shape, dtype, pool=None):
        self.shape, self.dtype, self.pool, self.device = tuple(shape), dtype, pool, "none"

    def get_device(self):
        return 0

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def is_contiguous(self):
        return True

    def numel(self):
        return int(np.prod(self.shape))

    def data_ptr(self):
        return A

    def record_stream(self, stream):
        pass


def _fake_torch_streams(monkeypatch, made):
    """torch.empty notes the stream that is current when it allocates; torch.cuda.stream switches it."""
    import contextlib

    import torch
    now = ["current"]

    @contextlib.contextmanager
    def switch(stream):
        before, now[0] = now[0], now[0] if stream is None else stream
        yield
        now[0] = before

    def empty(*shape, dtype=None, device=None):
        made.append(_Buffer(shape, dtype, now[0]))
        return made[-1]

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", switch)


def test_attention_allocates_its_workspace_on_its_stream(L, monkeypatch):
    """A workspace that a call makes itself comes from the pool of the stream that it runs on: one from the current
    stream's pool may still be in use by kernels there, for which the other stream does not wait."""
    import torch
    from paper_2609_29505_amd import binding
    made, calls = [], []
    lib = binding.lib()

    class Fake:
        sgd_op_attention_ranges_bytes = lib.sgd_op_attention_ranges_bytes

        @staticmethod
        def sgd_op_attention_ranges(dt, call, ws, nbytes, st):
            calls.append((ws, nbytes, st))
            return 0

    _fake_torch_streams(monkeypatch, made)
    monkeypatch.setattr(binding, "lib", lambda: Fake)
    monkeypatch.setattr(binding, "_here", lambda stream: (0, 5 if stream is None else 7))
    q, k = _Buffer((1, 1, 8, 128), torch.bfloat16), _Buffer((1, 4096, 2, 128), torch.bfloat16)
    r = _Buffer((1, 1, 2), torch.int32)
    for stream in (None, "other"):
        P.op_attention_ranges(q, k, k, q, r, stream=stream)
    assert [b.pool for b in made] == ["current", "other"] and [c[2] for c in calls] == [5, 7]
    assert all(c[1] == b.numel() > 0 for c, b in zip(calls, made))


@pytest.mark.parametrize("call", ["group_norm", "matrix_stats", "schedule_build"])
def test_calls_allocate_their_scratch_on_their_stream(L, monkeypatch, call):
    """As the attention's workspace: the scratch of the older calls that make their own."""
    import torch
    from paper_2609_29505_amd import binding
    made, calls = [], []

    class Fake:
        def __getattr__(self, name):
            def f(*args):
                if name.endswith("bytes"):
                    args[-1]._obj.value = 4096
                else:
                    calls.append(name)
                return 0
            return f

    _fake_torch_streams(monkeypatch, made)
    fake = Fake()
    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 5 if stream is None else 7)
    x = _Buffer((2, 4, 32), torch.bfloat16)
    w = _Buffer((8, 8), torch.float32)
    w.is_cuda, w.dim = True, lambda: 2
    for stream in (None, "other"):
        if call == "group_norm":
            P.op_group_norm_silu(x, x, 4, x, x, stream=stream)
        elif call == "matrix_stats":
            P.matrix_stats(w, stream=stream)
        else:
            P.schedule_build([[("w1", w)]], [1], 4, stream=stream)
    assert len(calls) == 2 and [b.pool for b in made] == ["current", "other"]


@pytest.mark.parametrize("dt,change,code", [
    (0, dict(scale=1.0, cap=2.0 ** 126), 0), (0, dict(cap=2.0 ** 126), ARG), (0, dict(scale=2.0, cap=1.01 * 2.0 ** 126), ARG), (0, dict(scale=8.0, cap=3e38), ARG), (0, dict(scale=2.0 ** 126), 0),
    (0, dict(scale=3e38), ARG), (1, dict(scale=3e38), ARG), (0, dict(scale=1e-39), ARG), (1, dict(scale=2.0 ** -126), 0),
    (0, dict(scale=1e-3, cap=1e37), ARG), (0, dict(scale=2.0 ** 126, cap=1.0), ARG), (0, dict(scale=2.0 ** 126, cap=2.0 ** 126), 0)])
def test_attention_scale_and_cap_limits(L, dt, change, code):
    """Past them fp32's products with log2(e) are infinite (a score of zero would come out NaN) or lose bits."""
    n = C.c_size_t()
    rc = L.sgd_op_attention_ranges_bytes(dt, C.byref(_call(**change)), C.byref(n))
    assert rc == code, (rc, L.sgd_last_error())


@pytest.mark.parametrize("change", [dict(scale=1e-60), dict(cap=1e-60), dict(scale=0.0), dict(scale=math.nan)])
def test_attention_refuses_what_fp32_holds_as_zero(L, monkeypatch, change):
    """The library takes scale 0 for the default and cap 0 for none."""
    import torch
    from paper_2609_29505_amd import binding
    monkeypatch.setattr(binding, "_here", lambda stream: (0, 5))
    q, k, r = _Buffer((1, 1, 8, 128), torch.bfloat16), _Buffer((1, 64, 2, 128), torch.bfloat16), _Buffer((1, 1, 2), torch.int32)
    with pytest.raises(ValueError):
        P.op_attention_ranges(q, k, k, q, r, **change)


def test_replay_search_allocates_its_buffer_on_its_stream(L, monkeypatch):
    import types

    from paper_2609_29505_amd import binding
    made, calls = [], []

    class Fake:
        @staticmethod
        def sgd_replay_bytes(h, n):
            n._obj.value = 4096
            return 0

        @staticmethod
        def sgd_replay_search(*args):
            calls.append(args)
            return 0

    _fake_torch_streams(monkeypatch, made)
    monkeypatch.setattr(binding, "lib", lambda: Fake)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 5 if stream is None else 7)
    model = types.SimpleNamespace(n_units=2, cfg=types.SimpleNamespace(T=3), h=None, _args=lambda alpha, beta: binding.sgd_step_args())
    for stream in (None, "other"):
        binding.DeviceModel.replay_search(model, _Buffer((4,), None), stream=stream)
    assert len(calls) == 2 and [b.pool for b in made] == ["current", "other"]
