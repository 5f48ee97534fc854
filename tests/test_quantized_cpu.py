"""Refusals of the operators on quantised rows: what their C entry points and their binding turn down before anything
reaches a GPU."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2608_03065_amd import psc  # noqa: E402

INVALID = -1
BUF = C.create_string_buffer(4096)
AT = (C.addressof(BUF) + 255) // 256 * 256
NAN = float("nan")


def refused(status, name):
    return status == INVALID and name.encode() + b":" in psc.lib().psc_last_error()


def quantize(x=AT, dtype=1, x_stride=64, n=2, D=64, q=AT, q_stride=32, scales=AT, s_stride=4):
    return psc.lib().psc_quantize_mx(x, dtype, x_stride, n, D, q, q_stride, scales, s_stride, None)


@pytest.mark.parametrize("wrong", [dict(dtype=2), dict(n=-1), dict(D=-1), dict(x=None), dict(q=None), dict(scales=None), dict(q_stride=40),
                                   dict(q_stride=16), dict(q=AT + 8), dict(x=AT + 1), dict(x_stride=-1), dict(n=1 << 31), dict(s_stride=2),
                                   dict(s_stride=0), dict(scales=AT + 2), dict(D=(1 << 30) + 1)])
def test_quantize_mx_refuses(wrong):
    assert refused(quantize(**wrong), "psc_quantize_mx")


def lookup(form=3, q=AT, q_stride=32, scales=AT, s_stride=4, rows=5, D=64, ids=AT, n=2, out=AT, dtype=1, stride=64):
    return psc.lib().psc_lookup_rows(form, q, q_stride, scales, s_stride, rows, D, ids, n, out, dtype, stride, None)


@pytest.mark.parametrize("wrong", [dict(form=0), dict(form=1), dict(form=4), dict(q=None), dict(scales=None), dict(out=None), dict(q_stride=24),
                                   dict(q_stride=16), dict(q=AT + 4), dict(s_stride=3), dict(s_stride=0), dict(scales=AT + 1), dict(rows=-1),
                                   dict(D=-1), dict(n=-1), dict(dtype=2), dict(stride=63), dict(out=AT + 1), dict(ids=AT + 2),
                                   dict(ids=None, n=6), dict(n=1 << 31), dict(rows=1 << 31), dict(D=(1 << 30) + 1),
                                   dict(form=2), dict(form=2, q_stride=64, scales=AT + 2), dict(form=2, q_stride=64, scales=None)])
def test_lookup_rows_refuses(wrong):
    assert refused(lookup(**wrong), "psc_lookup_rows")


def norm(x=AT, x_dtype=1, x_stride=64, residual=AT, r_dtype=0, r_stride=64, n=2, D=64, gain=AT, eps=1e-6, to=1, out=AT, o_stride=64,
         scales=AT, s_stride=4):
    return psc.lib().psc_add_rms_norm(x, x_dtype, x_stride, residual, r_dtype, r_stride, n, D, gain, eps, to, out, o_stride, scales, s_stride,
                                      None)


@pytest.mark.parametrize("wrong", [dict(x=None), dict(x_dtype=2), dict(r_dtype=2), dict(x_stride=-1), dict(x=AT + 1), dict(r_stride=63),
                                   dict(residual=AT + 2), dict(n=-1), dict(D=-1), dict(n=1 << 31), dict(D=(1 << 30) + 1), dict(gain=AT + 2),
                                   dict(eps=-1.0), dict(eps=NAN), dict(to=4), dict(to=-1), dict(out=None), dict(out=AT + 1), dict(o_stride=63),
                                   dict(to=2, scales=None), dict(to=2, o_stride=72), dict(to=2, o_stride=48), dict(to=2, out=AT + 8),
                                   dict(to=2, scales=AT + 1), dict(to=3, scales=None), dict(to=3, o_stride=40), dict(to=3, o_stride=16),
                                   dict(to=3, s_stride=2), dict(to=3, scales=AT + 1), dict(to=3, out=AT + 8)])
def test_add_rms_norm_refuses(wrong):
    assert refused(norm(**wrong), "psc_add_rms_norm")


def head(x=AT, x_form=1, x_stride=64, x_scales=AT, xs_stride=4, B=2, D=64, states=1, w=AT, w_stride=32, w_scales=AT, ws_stride=4, V=8, bias=None,
         y=AT, dtype=1, stride=8, ws=AT, ws_bytes=1 << 40):
    return psc.lib().psc_head_logits_mx(x, x_form, x_stride, x_scales, xs_stride, B, D, states, w, w_stride, w_scales, ws_stride, V, bias, None,
                                        y, dtype, stride, ws, ws_bytes, None)


@pytest.mark.parametrize("wrong", [dict(x_form=2), dict(x_form=4), dict(x_form=3), dict(states=0), dict(states=2), dict(states=4), dict(dtype=-1),
                                   dict(B=-1), dict(V=-1), dict(D=0), dict(D=131073), dict(x=None), dict(w=None), dict(w_scales=None),
                                   dict(y=None), dict(ws=None), dict(w_stride=40), dict(w_stride=16), dict(w_stride=1 << 22), dict(w=AT + 8),
                                   dict(ws_stride=2), dict(ws_stride=6), dict(ws_stride=1 << 22), dict(w_scales=AT + 2), dict(x=AT + 1),
                                   dict(y=AT + 1), dict(stride=7), dict(ws_bytes=263), dict(ws=AT + 8), dict(x_stride=-64),
                                   dict(x_form=3, states=3, x_stride=40), dict(x_form=3, states=3, x_stride=16),
                                   dict(x_form=3, states=3, x_stride=32, x=AT + 8), dict(x_form=3, states=3, x_stride=32, x_scales=None),
                                   dict(x_form=3, states=3, x_stride=32, xs_stride=1)])
def test_head_logits_mx_refuses(wrong):
    assert refused(head(**wrong), "psc_head_logits_mx")


def head_i8(q=AT, q_stride=64, scales=AT, B=2, D=64, w=AT, w_stride=64, w_scales=AT, V=8, y=AT, dtype=1, stride=8, ws=AT, ws_bytes=1 << 40):
    return psc.lib().psc_head_logits_quantized(q, q_stride, scales, B, D, w, w_stride, w_scales, V, None, None, y, dtype, stride, ws, ws_bytes, None)


@pytest.mark.parametrize("wrong", [dict(q=None), dict(scales=None), dict(q_stride=72), dict(q_stride=48), dict(q=AT + 8), dict(scales=AT + 2),
                                   dict(B=-1), dict(V=-1), dict(D=0), dict(D=131073), dict(w=None), dict(w_scales=None), dict(y=None),
                                   dict(ws=None), dict(w_stride=60), dict(stride=7), dict(ws_bytes=263), dict(dtype=2)])
def test_head_logits_i8_refuses(wrong):
    assert refused(head_i8(**wrong), "psc_head_logits_quantized")


def test_sizes_that_pass_a_launch_or_its_offsets_are_refused():
    V = (1 << 26) + 1
    assert psc.lib().psc_head_mx_workspace(2, 64, V, 1) == 0 and psc.lib().psc_head_mx_workspace(2, 64, 8, 0) == 0
    assert refused(head(V=V, stride=V), "psc_head_logits_mx") and b"2^26" in psc.lib().psc_last_error()
    most = ((1 << 23) - 1) * 64
    for B, V in ((most + 1, 8), (most // 2 + 64, 513), ((1 << 31) - 1, 1)):
        assert refused(head(B=B, V=V, stride=V), "psc_head_logits_mx") and b"2^23" in psc.lib().psc_last_error()
    # the last ones that are taken get as far as the workspace's check
    for B, V in ((2, 1 << 26), (most, 512), (64 * 63, 1 << 26)):
        assert refused(head(B=B, V=V, stride=V, ws_bytes=1), "psc_head_logits_mx") and b"workspace" in psc.lib().psc_last_error()


def test_head_mx_workspace_holds_states():
    L = psc.lib()
    assert L.psc_head_mx_workspace(3, 64, 8, 1) >= 3 * 512 and L.psc_head_mx_workspace(65535, 131072, 8, 1) >= 65535 * 262144
    assert L.psc_head_mx_workspace(65535, 131072, 8, 3) >= 65535 * (65536 + 4096)


def test_empty_calls_are_no_ops():
    assert quantize(n=0, x=None, q=None, scales=None) == 0 and quantize(D=0, x=None, q=None) == 0
    assert lookup(n=0, q=None, out=None) == 0 and lookup(D=0, q=None, out=None) == 0
    assert norm(n=0, x=None, out=None) == 0 and norm(D=0, x=None, out=None) == 0
    assert head(B=0, x=None, ws=None) == 0 and head(V=0, w=None, y=None) == 0
    assert head_i8(B=0, q=None, ws=None) == 0 and head_i8(V=0, w=None, y=None) == 0


def test_the_binding_refuses_tensors_that_the_library_cannot_check():
    """Host tensors, other types and other shapes never reach the library."""
    x, q, s = torch.zeros(2, 64), torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8)
    for call in (lambda: psc.quantize_mx(x), lambda: psc.quantize_mx(x.half()), lambda: psc.quantize_mx(x[0]),
                 lambda: psc.lookup_rows(q, s), lambda: psc.lookup_rows(x, s), lambda: psc.lookup_rows(q[0], s),
                 lambda: psc.add_rms_norm(x), lambda: psc.add_rms_norm(x, to="fp8"), lambda: psc.add_rms_norm(None),
                 lambda: psc.head_logits_mx(x, q, s), lambda: psc.head_logits_mx(x, q, s, states="i8"),
                 lambda: psc.head_logits_mx(q, q, s, x_scales=s), lambda: psc.head_logits(q, q, s, x_scales=s)):
        with pytest.raises(ValueError):
            call()


def test_the_binding_refuses_a_d_that_is_not_the_states():
    q, s = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8)
    for D in (0, 1, 62, 65, 128, -1):
        with pytest.raises(ValueError, match="x of"):
            psc.head_logits_mx(q, q, s, x_scales=s, D=D)
    for D in (63, 64):                  # taken: what is refused is that they are host tensors
        with pytest.raises(ValueError, match="device"):
            psc.head_logits_mx(q, q, s, x_scales=s, D=D)
