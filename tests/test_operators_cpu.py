"""Refusals of the operators around the logits: what their C entry points and
their binding turn down before anything reaches a GPU."""
import ctypes as C
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

from paper_2608_03065_amd import psc  # noqa: E402

INVALID = -1
BUF = C.create_string_buffer(4096)
AT = (C.addressof(BUF) + 255) // 256 * 256


def quantize(x=AT, dtype=1, x_stride=64, n=2, D=64, q=AT, q_stride=64, scales=AT):
    return psc.lib().psc_quantize_rows(x, dtype, x_stride, n, D, q, q_stride, scales, None)


@pytest.mark.parametrize("wrong", [dict(dtype=2), dict(n=-1), dict(D=-1), dict(x=None), dict(q=None),
                                   dict(scales=None), dict(q_stride=72), dict(q_stride=48), dict(q=AT + 8),
                                   dict(x=AT + 1), dict(x_stride=-1), dict(n=1 << 31)])
def test_quantize_rows_refuses(wrong):
    assert quantize(**wrong) == INVALID and b"psc_quantize_rows" in psc.lib().psc_last_error()


def head(x=AT, x_dtype=1, x_stride=64, B=2, D=64, w=AT, w_stride=64, w_scales=AT, V=8, y=AT, dtype=1, stride=8, ws=AT,
         ws_bytes=1 << 20):
    return psc.lib().psc_head_logits(x, x_dtype, x_stride, B, D, w, w_stride, w_scales, V, None, None, y, dtype, stride,
                                     ws, ws_bytes, None)


@pytest.mark.parametrize("wrong", [dict(x_dtype=2), dict(dtype=-1), dict(B=-1), dict(V=-1), dict(D=0), dict(D=131073),
                                   dict(x=None), dict(w=None), dict(w_scales=None), dict(y=None), dict(ws=None),
                                   dict(w_stride=60), dict(w_stride=48), dict(w_stride=1 << 22), dict(w=AT + 8),
                                   dict(x=AT + 1), dict(y=AT + 1), dict(stride=7), dict(ws_bytes=263), dict(ws=AT + 8),
                                   dict(x_stride=-64)])
def test_head_logits_refuses(wrong):
    assert head(**wrong) == INVALID and b"psc_head_logits" in psc.lib().psc_last_error()


def test_head_workspace_holds_states_and_scales():
    L = psc.lib()
    assert L.psc_head_workspace(0, 64, 8) == 0
    assert L.psc_head_workspace(3, 64, 8) >= 3 * (64 + 4) and L.psc_head_workspace(65535, 131072, 8) >= 65535 * 131076


def penalize(B=2, V=8, dtype=0, stride=8, logits=AT, **fields):
    p = psc._Penalties(**dict(dict(history=AT, lens=AT, cap=4, n_bias=1, bias_ids=AT, bias_values=AT), **fields))
    return psc.lib().psc_penalize(logits, dtype, stride, B, V, C.byref(p), None, None)


@pytest.mark.parametrize("wrong", [dict(dtype=3), dict(B=-1), dict(V=-1), dict(logits=None), dict(stride=7),
                                   dict(logits=AT + 2), dict(cap=-1), dict(cap=(1 << 30) + 1), dict(history=None),
                                   dict(lens=None), dict(n_bias=-1), dict(n_bias=1025), dict(bias_ids=None),
                                   dict(bias_values=None)])
def test_penalize_refuses(wrong):
    assert penalize(**wrong) == INVALID and b"psc_penalize" in psc.lib().psc_last_error()


def append(history=AT, cap=4, lens=AT, B=2, tokens=AT):
    return psc.lib().psc_append_tokens(history, cap, lens, B, tokens, None, None)


@pytest.mark.parametrize("wrong", [dict(history=None), dict(cap=-1), dict(lens=None), dict(B=-1), dict(tokens=None)])
def test_append_tokens_refuses(wrong):
    assert append(**wrong) == INVALID and b"psc_append_tokens" in psc.lib().psc_last_error()


def sample(logits=AT, dtype=0, stride=8, B=2, V=8, k=4, tokens=AT, ws=AT, ws_bytes=1 << 20):
    return psc.lib().psc_sample(logits, dtype, stride, B, V, None, None, k, tokens, None, None, None, ws, ws_bytes, None)


@pytest.mark.parametrize("wrong", [dict(logits=None), dict(dtype=2), dict(stride=7), dict(B=-1), dict(B=65536), dict(V=-1),
                                   dict(V=0), dict(k=0), dict(k=65), dict(tokens=None), dict(ws=None), dict(ws=AT + 8),
                                   dict(ws_bytes=1), dict(logits=AT + 2), dict(V=1 << 20, stride=1 << 20)])
def test_sample_refuses(wrong):
    assert sample(**wrong) == INVALID and b"psc_sample" in psc.lib().psc_last_error()


def test_empty_batches_are_no_ops():
    assert quantize(n=0, x=None, q=None, scales=None) == 0
    assert head(B=0, x=None, ws=None) == 0 and head(V=0, w=None, y=None) == 0
    assert penalize(B=0, logits=None) == 0 and penalize(V=0, logits=None) == 0
    assert append(B=0, history=None, lens=None, tokens=None) == 0
    assert sample(B=0, logits=None, tokens=None, ws=None) == 0


def test_the_binding_refuses_tensors_that_the_library_cannot_check():
    """Host tensors, other types and other shapes never reach the library."""
    x = torch.zeros(2, 64)
    for call in (lambda: psc.quantize_rows(x), lambda: psc.head_logits(x, x.to(torch.int8), x[:, 0]),
                 lambda: psc.penalize(x), lambda: psc.sample(x, 4), lambda: psc.quantize_rows(x.half()),
                 lambda: psc.quantize_rows(x[0]), lambda: psc.sample(x.t(), 4), lambda: psc.penalize(None),
                 lambda: psc.append_tokens(x, x, x)):
        with pytest.raises(ValueError):
            call()


def test_head_logits_refuses_vocabularies_whose_masks_pass_32_bit_offsets():
    V = (1 << 26) + 1
    assert psc.lib().psc_head_workspace(2, 64, V) == 0
    assert head(V=V, stride=V) == INVALID and b"2^26" in psc.lib().psc_last_error()
    # the last one that is taken gets as far as the workspace's check
    assert head(V=V - 1, stride=V, ws_bytes=1) == INVALID and b"workspace" in psc.lib().psc_last_error()


def test_sample_refuses_rows_past_two_mib_less_a_line():
    most = ((2 << 20) - 128) // 2
    assert sample(dtype=1, V=most + 2, stride=most + 2, ws_bytes=1) == INVALID and b"2 MiB" in psc.lib().psc_last_error()
    assert sample(dtype=1, V=most, stride=most, ws_bytes=1) == INVALID and b"workspace" in psc.lib().psc_last_error()
    # sizes in bytes that pass 32 bits
    for V in (1 << 29, 1 << 30, (1 << 31) - 1):
        for dtype in (0, 1):
            assert sample(dtype=dtype, V=V, stride=V) == INVALID and b"2 MiB" in psc.lib().psc_last_error()


def test_head_logits_refuses_more_tiles_than_a_launch_holds():
    most = ((1 << 24) - 1) * 64
    for B, V in ((most + 1, 8), (most + 1, 512), (most // 2, 513), ((1 << 31) - 1, 1)):
        assert head(B=B, V=V, stride=V, ws_bytes=1 << 62) == INVALID and b"2^24" in psc.lib().psc_last_error()
    # the last one that is taken gets as far as the workspace's check
    for B, V in ((most, 512), (((1 << 23) - 1) * 64, 1024), (64, 1 << 26)):
        assert head(B=B, V=V, stride=V, ws_bytes=1) == INVALID and b"workspace" in psc.lib().psc_last_error()


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no device's: every launch has to fail")
def test_penalize_ends_after_the_last_of_the_most_rows():
    """Rows are dealt over launches; the number of those done passes 31 bits after the last ones of 2^31 - 1."""
    code = ("from paper_2608_03065_amd import psc; import ctypes as C; at = C.addressof(C.create_string_buffer(64)); "
            "assert psc.lib().psc_penalize(at, 0, 1, 2**31 - 1, 1, None, at, None) == -5")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert subprocess.run([sys.executable, "-c", code], cwd=root, timeout=60).returncode == 0
