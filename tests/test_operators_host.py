"""What the operators refuse before they touch a GPU: the C entry points, called with addresses that are never read."""
import ctypes

import pytest

import paper_2406_06237_b200 as ans
from paper_2406_06237_b200 import binding as B

INVALID, UNSUPPORTED, TOO_SMALL = ans.ANS_ERR_INVALID_ARG, ans.ANS_ERR_UNSUPPORTED, ans.ANS_ERR_BUFFER_TOO_SMALL
P = 1 << 20                                              # an address on every boundary asked for


def norm(**kw):
    d = B.ans_norm_desc(d_x=P, d_out=P, d_scales=P, rows=4, x_stride=64, residual_stride=64, out_stride=64, sum_stride=64, width=64, eps=1e-6,
                        x_dtype=ans.ANS_BF16, weight_dtype=ans.ANS_BF16, out_dtype=ans.ANS_E4M3)
    for k, v in kw.items():
        setattr(d, k, v)
    return ans.lib().ans_rms_norm(d, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(d_x=None), INVALID), (dict(d_out=None), INVALID), (dict(d_scales=None), INVALID), (dict(d_x=P + 1), INVALID),
    (dict(x_stride=63), INVALID), (dict(out_stride=10), INVALID), (dict(d_residual=P, residual_stride=0), INVALID), (dict(d_sum=P, sum_stride=8), INVALID),
    (dict(d_weight=P + 1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(x_dtype=ans.ANS_U8), UNSUPPORTED), (dict(x_dtype=ans.ANS_E4M3), UNSUPPORTED), (dict(out_dtype=ans.ANS_U8), UNSUPPORTED),
    (dict(weight_dtype=7), UNSUPPORTED), (dict(width=32769, x_stride=40000, out_stride=40000), UNSUPPORTED),
    (dict(rows=0, d_x=None), 0), (dict(width=0, d_out=None), 0)])
def test_norm(kw, rc):
    assert norm(**kw) == rc


def product(status=P, **kw):
    d = B.ans_product_desc(d_x=P, d_w=P, d_y=P, x_stride=64, w_stride=64, residual_stride=32, y_stride=32, m=4, n=32, k=64, dtype=ans.ANS_BF16,
                           y_dtype=ans.ANS_BF16)
    for k, v in kw.items():
        setattr(d, k, v)
    return ans.lib().ans_product(d, status, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(d_x=None), INVALID), (dict(d_w=None), INVALID), (dict(d_y=None), INVALID), (dict(status=None), INVALID), (dict(d_x=P + 8), TOO_SMALL), (dict(d_x=P + 1), INVALID),
    (dict(d_w=P + 2), INVALID), (dict(d_y=P + 1), INVALID), (dict(d_residual=P + 1), INVALID), (dict(d_bias=P + 2), INVALID), (dict(x_stride=63), INVALID),
    (dict(x_stride=68), TOO_SMALL), (dict(x_stride=68, d_room=P, room_bytes=4 * 128 - 1), TOO_SMALL), (dict(x_stride=68, d_room=P + 8, room_bytes=512), INVALID), (dict(w_stride=0), INVALID), (dict(y_stride=31), INVALID), (dict(d_residual=P, residual_stride=5), INVALID),
    (dict(dtype=ans.ANS_F32), UNSUPPORTED), (dict(y_dtype=ans.ANS_E4M3), UNSUPPORTED), (dict(activation=5), UNSUPPORTED), (dict(activation=-1), UNSUPPORTED),
    (dict(flags=2), UNSUPPORTED), (dict(k=(1 << 22) + 1), UNSUPPORTED), (dict(m=(1 << 30) + 1), UNSUPPORTED), (dict(m=0, d_x=None), 0), (dict(n=0, d_w=None), 0)])
def test_product(kw, rc):
    assert product(**kw) == rc


def test_product_room():
    def room(**kw):
        d = B.ans_product_desc(d_x=P, x_stride=64, m=4, k=64, dtype=ans.ANS_BF16)
        for k, v in kw.items():
            setattr(d, k, v)
        return ans.binding.ans_product_room_bytes(d)
    assert room() == room(m=1, x_stride=3) == room(dtype=ans.ANS_E4M3) == 0
    assert room(x_stride=65) == room(d_x=P + 2) == 4 * 128 and room(x_stride=65, k=61) == 4 * 128 and room(x_stride=65, k=56) == 4 * 112
    assert room(dtype=ans.ANS_E4M3, x_stride=65, k=33) == 4 * 48
    with pytest.raises(ans.AnsError):
        room(dtype=ans.ANS_U8)
    assert ans.lib().ans_product_room_bytes(None, None) == INVALID


def cache_desc(**kw):
    d = B.ans_cache_desc(d_k_codes=P, d_k_scales=P, d_k_zeros=P, d_v_codes=P, d_v_scales=P, d_v_zeros=P, n_pages=4, page_size=16, heads=2, head_dim=64,
                         group=64, bitwidth=8)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


CACHE = [(dict(bitwidth=2), UNSUPPORTED), (dict(group=8), UNSUPPORTED), (dict(group=24), UNSUPPORTED), (dict(group=512, head_dim=512), UNSUPPORTED),
         (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(heads=0), INVALID), (dict(page_size=0), INVALID),
         (dict(d_k_codes=None), INVALID), (dict(d_v_zeros=None), INVALID), (dict(d_v_codes=P + 8), INVALID), (dict(d_k_scales=P + 4), INVALID),
         (dict(heads=1 << 16), UNSUPPORTED)]


@pytest.mark.parametrize("kw,rc", CACHE)
def test_cache(kw, rc):
    d = cache_desc(**kw)
    assert ans.lib().ans_cache_write(d, P, P, ans.ANS_BF16, 3, 128, 64, 128, 64, P, P, None) == rc
    assert ans.lib().ans_cache_read(d, P, 4, 4, 1, P, 3, P, P, ans.ANS_BF16, P, None) == rc


def test_cache_write():
    w = lambda k=P, v=P, dt=ans.ANS_BF16, n=3, s=(128, 64, 128, 64), slots=P, status=P: ans.lib().ans_cache_write(cache_desc(), k, v, dt, n, *s, slots, status, None)  # noqa: E731
    assert w(k=None) == w(v=None) == w(slots=None) == w(status=None) == w(k=P + 1) == w(slots=P + 4) == INVALID
    assert w(dt=ans.ANS_E4M3) == w(dt=ans.ANS_U8) == w(n=1 << 41) == w(s=(1 << 41, 0, 0, 0)) == UNSUPPORTED
    assert w(k=None, n=0) == 0


def test_cache_read():
    def r(tables=P, stride=4, pages=4, n=2, starts=P, rows=3, k=P, v=P, dt=ans.ANS_BF16, status=P):
        return ans.lib().ans_cache_read(cache_desc(), tables, stride, pages, n, starts, rows, k, v, dt, status, None)
    assert r(tables=None) == r(starts=None) == r(k=None) == r(v=None) == r(status=None) == r(k=P + 8) == r(starts=P + 2) == r(stride=3) == INVALID
    assert r(dt=ans.ANS_E4M3) == r(rows=1 << 31) == UNSUPPORTED
    assert r(rows=0, k=None) == r(n=0, tables=None) == 0


def test_descriptors_have_the_header_layout(tmp_path):
    """Sizes and last fields' places of the ctypes structures against the C compiler's."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    c = tmp_path / "sizes.c"
    c.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ans_b200.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(ans_norm_desc), '
                 "offsetof(ans_norm_desc, out_dtype), sizeof(ans_product_desc), offsetof(ans_product_desc, room_bytes), sizeof(ans_cache_desc), "
                 "offsetof(ans_cache_desc, bitwidth)); return 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), "-o", str(tmp_path / "sizes"), str(c)])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "sizes")]).split()]
    assert got == [ctypes.sizeof(B.ans_norm_desc), B.ans_norm_desc.out_dtype.offset, ctypes.sizeof(B.ans_product_desc), B.ans_product_desc.room_bytes.offset,
                   ctypes.sizeof(B.ans_cache_desc), B.ans_cache_desc.bitwidth.offset]


def test_a_handle_needs_a_gpu():
    import torch

    from paper_2406_06237_b200.runtime import Linear, PagedCache, RmsNorm
    for make in (lambda: RmsNorm(torch.ones(4)), lambda: Linear(torch.ones(4, 4, dtype=torch.bfloat16)), lambda: PagedCache(1, 1, 1, 16, device="cpu")):
        with pytest.raises(RuntimeError):
            make()


def test_forms():
    """The module that spares a repeated call its checks: any change of type, size, stride or presence is seen."""
    import torch

    from paper_2406_06237_b200._ans_form import Form
    f, a, b = Form(), torch.zeros(4, 6), torch.zeros(3, dtype=torch.int64)
    assert f.places(a, b) is None
    f.keep(a, None, b)
    assert f.places(a, None, b) == (a.data_ptr(), 0, b.data_ptr())
    other = torch.ones(4, 6)
    assert f.places(other, None, b)[0] == other.data_ptr()
    for args in ((a, b), (a, None, b, b), (a, a, b), (None, None, b), (a.double(), None, b), (a.t(), None, b), (a[:, :5], None, b), (a[:3], None, b),
                 (a.view(6, 4), None, b), (a[None], None, b), (a, None, b.int()), (a.view(4, 6)[:, ::2], None, b), ()):
        assert f.places(*args) is None
    with pytest.raises(TypeError):
        f.places(a, 3, b)
    with pytest.raises(TypeError):
        f.keep("x")
    f.keep()
    assert f.places(a, None, b) is None and f.places() is None
