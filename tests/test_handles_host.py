"""What the handles and the entry points behind them refuse before they touch a GPU."""
import pytest

import paper_2406_06237_b200 as ans

INVALID, UNSUPPORTED, TOO_SMALL = ans.ANS_ERR_INVALID_ARG, ans.ANS_ERR_UNSUPPORTED, ans.ANS_ERR_BUFFER_TOO_SMALL
P = 1 << 20                                              # an address on every boundary asked for; never read


@pytest.mark.parametrize("kw,rc", [
    (dict(d_from=None), INVALID), (dict(d_to=None), INVALID), (dict(d_from=P + 1), INVALID), (dict(d_to=P + 8), INVALID),
    (dict(dtype=ans.ANS_F32), UNSUPPORTED), (dict(dtype=ans.ANS_U8), UNSUPPORTED), (dict(rows=(1 << 30) + 1), UNSUPPORTED),
    (dict(k=(1 << 22) + 1), UNSUPPORTED), (dict(stride=1 << 37), UNSUPPORTED), (dict(step=1 << 37), UNSUPPORTED),
    (dict(rows=1 << 30, k=1 << 22), UNSUPPORTED), (dict(rows=0, d_from=None), 0), (dict(k=0, d_to=None), 0)])
def test_product_rows(kw, rc):
    a = {**dict(d_from=P, stride=65, step=1, rows=4, k=65, dtype=ans.ANS_BF16, d_to=P), **kw}
    assert ans.lib().ans_product_rows(*(a[f] for f in ("d_from", "stride", "step", "rows", "k", "dtype", "d_to")), None) == rc


ANYWHERE = ans.binding.ANS_PRODUCT_WEIGHTS_ANYWHERE


@pytest.mark.parametrize("kw,rc", [
    (dict(d_w=P + 2), TOO_SMALL), (dict(w_stride=65), TOO_SMALL), (dict(w_stride=65, d_room=P, room_bytes=32 * 128 - 1), TOO_SMALL),
    (dict(w_stride=65, d_room=P + 8, room_bytes=1 << 20), INVALID), (dict(d_w=P + 1), INVALID), (dict(w_stride=63), INVALID),
    (dict(d_w=P + 2, x_stride=65, d_room=P, room_bytes=36 * 128 - 1), TOO_SMALL), (dict(flags=ANYWHERE | 2), UNSUPPORTED),
    (dict(d_w=P + 2, n=1 << 30, y_stride=1 << 30, k=1 << 22, x_stride=1 << 22, w_stride=1 << 22, d_room=P, room_bytes=1 << 62), UNSUPPORTED)])
def test_weights_anywhere(kw, rc):
    d = ans.binding.ans_product_desc(d_x=P, d_w=P, d_y=P, x_stride=64, w_stride=64, residual_stride=32, y_stride=32, m=4, n=32, k=64, dtype=ans.ANS_BF16,
                                     y_dtype=ans.ANS_BF16, flags=ANYWHERE)
    for k, v in kw.items():
        setattr(d, k, v)
    assert ans.lib().ans_product(d, P, None) == rc


def test_room_for_weights_anywhere():
    def room(**kw):
        d = ans.binding.ans_product_desc(d_x=P, d_w=P, x_stride=64, w_stride=64, m=4, n=32, k=64, dtype=ans.ANS_BF16, flags=ANYWHERE)
        for k, v in kw.items():
            setattr(d, k, v)
        return ans.binding.ans_product_room_bytes(d)
    assert room() == room(n=1, w_stride=65) == room(flags=0, d_w=P + 2) == 0
    assert room(d_w=P + 2) == room(w_stride=65) == 32 * 128 and room(w_stride=65, x_stride=65) == 36 * 128 and room(x_stride=65) == 4 * 128
    assert room(dtype=ans.ANS_E4M3, w_stride=65, k=33) == 32 * 48


def test_product_form():
    import ctypes
    d, t, p = ans.binding.ans_product_desc(m=3, n=4, k=5, dtype=ans.ANS_BF16), ctypes.c_uint32(), ctypes.c_uint32()
    f = ans.lib().ans_product_form
    assert f(None, ctypes.byref(t), ctypes.byref(p)) == f(d, None, ctypes.byref(p)) == f(d, ctypes.byref(t), None) == INVALID
    d.dtype = ans.ANS_F32
    assert f(d, ctypes.byref(t), ctypes.byref(p)) == UNSUPPORTED
    d.dtype, d.m = ans.ANS_E4M3, 0
    assert f(d, ctypes.byref(t), ctypes.byref(p)) == 0 and t.value == p.value == 0


def test_a_missing_or_foreign_module_says_what_to_run(monkeypatch):
    """Without the module of tensor forms, or with one of another torch or Python, a handle says so; nothing is guessed."""
    import sys
    import types

    import paper_2406_06237_b200 as package
    from paper_2406_06237_b200 import operators
    name = "paper_2406_06237_b200._ans_form"
    monkeypatch.delattr(package, "_ans_form", raising=False)
    monkeypatch.setitem(sys.modules, name, None)
    with pytest.raises(ImportError, match=r"build\.build\(\)"):
        operators._form_type()
    other = types.ModuleType(name)
    other.MADE_FOR, other.Form = "torch 1.0, cpython-27", object
    monkeypatch.setitem(sys.modules, name, other)
    with pytest.raises(ImportError, match=r"torch 1\.0.*build\.build\(\)"):
        operators._form_type()
    monkeypatch.undo()
    assert operators._form_type()().places() is None


def test_the_module_is_rebuilt_for_another_torch(monkeypatch, tmp_path):
    from paper_2406_06237_b200 import build
    binary, noted = tmp_path / "form.so", tmp_path / "made_for"
    monkeypatch.setattr(build, "FORM", str(binary))
    monkeypatch.setattr(build, "FORM_MADE_FOR", str(noted))
    assert not build.form_is_current()
    binary.write_bytes(b"")
    assert not build.form_is_current()                   # built by something that noted nothing
    noted.write_text("torch 1.0, cpython-27")
    assert not build.form_is_current()
    noted.write_text(build.form_interface())
    assert build.form_is_current()


def test_build_builds_both(monkeypatch):
    from paper_2406_06237_b200 import build
    asked = []
    monkeypatch.setattr(build, "build_form", lambda force=False: asked.append(force))
    monkeypatch.setattr(build, "sources", lambda: [])
    monkeypatch.setattr(build.subprocess, "check_call", lambda cmd: asked.append("nvcc"))
    build.build(force=True)
    assert asked == [True, "nvcc"]
