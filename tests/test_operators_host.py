"""What the operators around the step refuse, on the host before anything is launched (CPU only)."""
import ctypes as C
import os

import pytest
import torch

from paper_2602_21780_amd import xsv


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(xsv.LIB_PATH):
        from paper_2602_21780_amd.build import build
        build()
    return xsv.lib()


PTR = 1 << 20    # an aligned address that nothing looks at


def _rotate(**kw):
    good = dict(n=4, heads_q=2, heads_k=2, norm=2, axes=1, interleaved=0, eps=1e-5, base=100.0, positions=PTR, q_weight=None, q_bias=None,
                k_weight=None, k_bias=None)
    return xsv.xsv_rotate_config(**{**good, **kw})


T = xsv.xsv_tensor(PTR, 4 * 64, 64)
BAD_TENSORS = [xsv.xsv_tensor(None, 256, 64), xsv.xsv_tensor(PTR + 8, 256, 64), xsv.xsv_tensor(PTR, 256, 60), xsv.xsv_tensor(PTR, 256, 68),
               xsv.xsv_tensor(PTR, -256, 64), xsv.xsv_tensor(PTR, 4, 64), xsv.xsv_tensor(PTR, 256, (1 << 24) + 8)]


@pytest.mark.parametrize("bad", [dict(n=-1), dict(heads_q=-1), dict(heads_q=0, heads_k=0), dict(norm=3), dict(norm=-1), dict(axes=3), dict(axes=-1),
                                 dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(base=0.0),
                                 dict(base=float("nan")), dict(base=-2.0), dict(base=0.5), dict(base=float("inf")), dict(positions=None), dict(positions=PTR + 2), dict(q_weight=PTR + 1),
                                 dict(k_bias=PTR + 3)])
def test_rotate_refuses_bad_configurations(lib, bad):
    cfg = _rotate(**bad)
    nbytes = C.c_int64()
    assert lib.xsv_norm_rotate(None, C.byref(cfg), T, T, T, T) == xsv.XSV_ERR_ARG
    assert lib.xsv_norm_rotate_grad(None, C.byref(cfg), T, T, T, T, T, T, None, None, 0) == xsv.XSV_ERR_ARG
    assert lib.xsv_norm_rotate_grad_workspace(C.byref(cfg), C.byref(nbytes)) == xsv.XSV_ERR_ARG


def test_rotate_refuses_bad_tensors_and_workspaces(lib):
    cfg = _rotate()
    nbytes = C.c_int64()
    assert lib.xsv_norm_rotate(None, None, T, T, T, T) == xsv.XSV_ERR_ARG
    assert lib.xsv_norm_rotate_grad_workspace(C.byref(cfg), None) == xsv.XSV_ERR_ARG
    assert lib.xsv_norm_rotate_grad_workspace(C.byref(cfg), C.byref(nbytes)) == xsv.XSV_OK and nbytes.value > 0
    for bad in BAD_TENSORS:
        for at in range(4):
            ts = [T] * 4
            ts[at] = bad
            assert lib.xsv_norm_rotate(None, C.byref(cfg), *ts) == xsv.XSV_ERR_ARG
        for at in range(6):
            ts = [T] * 6
            ts[at] = bad
            assert lib.xsv_norm_rotate_grad(None, C.byref(cfg), *ts, None, None, 0) == xsv.XSV_ERR_ARG
    for sums, work, size in ((PTR, None, nbytes.value), (PTR, PTR, nbytes.value - 1), (PTR, PTR + 8, nbytes.value), (PTR + 2, PTR, nbytes.value)):
        assert lib.xsv_norm_rotate_grad(None, C.byref(cfg), T, T, T, T, T, T, sums, work, size) == xsv.XSV_ERR_ARG
    assert lib.xsv_norm_rotate(None, C.byref(_rotate(heads_q=(1 << 16) + 1)), T, T, T, T) == xsv.XSV_ERR_UNSUPPORTED
    empty = xsv.xsv_tensor(None, 0, 0)
    assert lib.xsv_norm_rotate(None, C.byref(_rotate(n=0, positions=None)), empty, empty, empty, empty) == xsv.XSV_OK    # nothing to do


def test_bindings_refuse_what_is_not_a_bf16_device_tensor():
    host = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    for call in (lambda: xsv.norm_rotate(host, host), lambda: xsv.norm_rotate_grad(host, host, host, host), lambda: xsv.norm_rotate(None)):
        with pytest.raises(ValueError):
            call()


def _seq(**kw):
    good = dict(heads=4, kv_heads=2, sequences=1, rows_q=8, rows_k=9, longest_q=8, longest_k=9, q_begin=PTR, k_begin=PTR, causal=0, softmax_scale=0.0)
    return xsv.xsv_seq_config(**{**good, **kw})


@pytest.mark.parametrize("bad", [dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(heads=-4), dict(sequences=-1), dict(rows_q=-1), dict(rows_k=-1),
                                 dict(longest_q=9), dict(longest_k=10), dict(longest_q=-1), dict(causal=-1), dict(softmax_scale=-1.0),
                                 dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(softmax_scale=1e-30), dict(softmax_scale=1e30), dict(q_begin=None), dict(k_begin=None),
                                 dict(q_begin=PTR + 2), dict(k_begin=PTR + 1)])
def test_seq_attend_refuses_bad_configurations(lib, bad):
    cfg = _seq(**bad)
    nbytes = C.c_int64()
    assert lib.xsv_seq_attend(None, C.byref(cfg), T, T, T, T, PTR, PTR, 1 << 20) == xsv.XSV_ERR_ARG
    assert lib.xsv_seq_attend_grad(None, C.byref(cfg), T, T, T, T, PTR, T, T, T, T, PTR, 1 << 20) == xsv.XSV_ERR_ARG
    assert lib.xsv_seq_attend_grad_workspace(C.byref(cfg), C.byref(nbytes)) == xsv.XSV_ERR_ARG
    assert lib.xsv_seq_attend_workspace(C.byref(cfg), C.byref(nbytes)) == xsv.XSV_ERR_ARG


def test_seq_attend_refuses_bad_tensors_workspaces_and_grids(lib):
    cfg = _seq()
    nbytes = C.c_int64()
    assert lib.xsv_seq_attend(None, None, T, T, T, T, PTR, PTR, 1 << 20) == xsv.XSV_ERR_ARG
    assert lib.xsv_seq_attend_grad_workspace(C.byref(cfg), None) == xsv.XSV_ERR_ARG
    assert lib.xsv_seq_attend_grad_workspace(C.byref(cfg), C.byref(nbytes)) == xsv.XSV_OK and nbytes.value >= 4 * 8 * 4
    for bad in BAD_TENSORS:
        for at in range(4):
            ts = [T] * 4
            ts[at] = bad
            assert lib.xsv_seq_attend(None, C.byref(cfg), *ts, PTR, PTR, 1 << 20) == xsv.XSV_ERR_ARG
        for at in range(8):
            ts = [T] * 8
            ts[at] = bad
            assert lib.xsv_seq_attend_grad(None, C.byref(cfg), *ts[:4], PTR, *ts[4:], PTR, nbytes.value) == xsv.XSV_ERR_ARG
    for lse in (None, PTR + 2):
        assert lib.xsv_seq_attend(None, C.byref(cfg), T, T, T, T, lse, PTR, 1 << 20) == xsv.XSV_ERR_ARG
        assert lib.xsv_seq_attend_grad(None, C.byref(cfg), T, T, T, T, lse, T, T, T, T, PTR, nbytes.value) == xsv.XSV_ERR_ARG
    for work, size in ((None, nbytes.value), (PTR + 8, nbytes.value), (PTR, nbytes.value - 1)):
        assert lib.xsv_seq_attend_grad(None, C.byref(cfg), T, T, T, T, PTR, T, T, T, T, work, size) == xsv.XSV_ERR_ARG
    long = _seq(rows_k=1000, longest_k=1000)      # few queries, many keys: workgroups share the keys
    assert lib.xsv_seq_attend_workspace(C.byref(long), C.byref(nbytes)) == xsv.XSV_OK and nbytes.value > 0
    for work, size in ((None, nbytes.value), (PTR + 8, nbytes.value), (PTR, nbytes.value - 1)):
        assert lib.xsv_seq_attend(None, C.byref(long), T, T, T, T, PTR, work, size) == xsv.XSV_ERR_ARG
    assert lib.xsv_seq_attend_workspace(C.byref(long), None) == xsv.XSV_ERR_ARG and lib.xsv_seq_attend_workspace(None, C.byref(nbytes)) == xsv.XSV_ERR_ARG
    huge = _seq(heads=1 << 16, kv_heads=1 << 16, rows_q=1 << 20, rows_k=1 << 20, longest_q=1 << 20, longest_k=1 << 20)
    assert lib.xsv_seq_attend(None, C.byref(huge), T, T, T, T, PTR, PTR, 1 << 20) == xsv.XSV_ERR_UNSUPPORTED


def test_seq_attend_binding_refuses_what_is_not_a_bf16_device_tensor():
    host = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    begin = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        xsv.seq_attend(host, host, host, begin)
    with pytest.raises(ValueError):
        xsv.seq_attend_grad(host, host, host, host, host, torch.zeros((2, 4)), begin)


class _Stream:
    cuda_stream, device = 1234, torch.device("cuda", 0)


def test_what_a_contexts_calls_allocate_belongs_to_the_stream_it_was_made_on(monkeypatch):
    """Without a stream= of its own a context keeps the one that is current when it is made; the library enqueues on that one later, too."""
    made, entered = [], []

    class Library:
        xsv_create = staticmethod(lambda cfg, stream, handle: made.append(stream) or xsv.XSV_OK)

    class Entered(Exception):
        pass

    def on(device, stream):
        entered.append(stream)
        raise Entered

    monkeypatch.setattr(xsv, "lib", lambda: Library)
    monkeypatch.setattr(xsv, "_on", on)
    monkeypatch.setattr(xsv, "_tensor", lambda *a, **kw: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream)
    ctx = xsv.Context(2, 2, 64, 8, 0, 0, 4, 64)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    assert made == [1234]
    x = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    for call in (lambda: ctx.query_attend(0, x), lambda: ctx.step(0, x, x, x), lambda: ctx.frame_attend(x, x, x), lambda: ctx.dequant_attend(0, x, x, x),
                 lambda: ctx.step_all_layers([x, x], [x, x], [x, x])):
        with pytest.raises(Entered):
            call()
    assert entered == [_Stream] * 5


@pytest.mark.parametrize("bad", [dict(longest_q=(1 << 32) + 5), dict(longest_k=(1 << 32) + 5), dict(causal=1 << 32), dict(causal=(1 << 32) + 1),
                                 dict(causal=1 << 31), dict(softmax_scale=1e-60), dict(softmax_scale=-1e-60)])
def test_seq_attend_binding_refuses_numbers_that_the_librarys_types_would_change(bad):
    """Bounds and blocks of 2^32 and more would arrive as small ones, and a scale too small for fp32 as 0, which asks for the usual scale."""
    x, begin = torch.zeros((2, 8, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    good = dict(longest_q=None, longest_k=None, causal=1, softmax_scale=0.0)
    assert xsv._seq_config(x, x, begin, None, **good).longest_q == 8
    with pytest.raises(ValueError):
        xsv._seq_config(x, x, begin, None, **{**good, **bad})
