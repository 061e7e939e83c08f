"""What the operators of a batch of requests refuse before they touch a GPU: the C entry points, called with addresses that
are never read."""
import ctypes

import pytest

import paper_2406_06237_b200 as ans
from paper_2406_06237_b200 import binding as B

INVALID, UNSUPPORTED, TOO_SMALL = ans.ANS_ERR_INVALID_ARG, ans.ANS_ERR_UNSUPPORTED, ans.ANS_ERR_BUFFER_TOO_SMALL
P = 1 << 20                                              # an address on every boundary asked for
FAR = (1 << 40) + 16


def changed(d, kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def pages(status=P, **kw):
    d = B.ans_pages_desc(d_cached=P, d_new=P, d_free=P, d_taken=P, d_tables=P, table_stride=8, table_pages=8, n_seqs=3, n_free=9, page_size=16, rows=5,
                         d_starts=P, d_lengths=P, d_ends=P, d_slots=P, d_positions=P, d_taken_out=P)
    return ans.lib().ans_page_tables(changed(d, kw), status, None)


@pytest.mark.parametrize("kw,rc", [
    *((dict([(f, None)]), INVALID) for f in ("d_cached", "d_new", "d_free", "d_taken", "d_tables", "d_starts", "d_lengths", "d_ends", "d_slots", "d_positions",
                                             "d_taken_out", "status")),
    *((dict([(f, P + 2)]), INVALID) for f in ("d_cached", "d_new", "d_free", "d_taken", "d_tables", "d_starts", "d_lengths", "d_ends", "d_positions", "d_taken_out")),
    (dict(d_slots=P + 4), INVALID), (dict(table_stride=7), INVALID), (dict(page_size=0), INVALID), (dict(page_size=(1 << 20) + 1), UNSUPPORTED),
    (dict(n_seqs=4097), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(table_stride=FAR), UNSUPPORTED), (dict(n_seqs=0, rows=0, d_starts=None), INVALID)])
def test_page_tables(kw, rc):
    assert pages(**kw) == rc


def adapters(status=P, **kw):
    d = B.ans_adapters_desc(d_x=P, d_y=P, d_out=2 * P, d_a=P, d_b=P, d_which=P, d_starts=P, x_stride=64, y_stride=32, out_stride=32, rows=4, n_seqs=2, count=3,
                            rank=8, n_in=64, n_out=32, x_dtype=ans.ANS_BF16, y_dtype=ans.ANS_BF16)
    return ans.lib().ans_adapters(changed(d, kw), status, None)


@pytest.mark.parametrize("kw,rc", [
    *((dict([(f, None)]), INVALID) for f in ("d_x", "d_y", "d_out", "d_a", "d_b", "d_which", "d_starts", "status")),
    *((dict([(f, P + 1)]), INVALID) for f in ("d_x", "d_y", "d_out", "d_a", "d_b")), *((dict([(f, P + 2)]), INVALID) for f in ("d_which", "d_starts", "d_scales", "d_x_scales")),
    (dict(y_dtype=ans.ANS_F32, d_y=P + 2), INVALID), (dict(x_stride=63), INVALID), (dict(y_stride=31), INVALID), (dict(out_stride=31), INVALID), (dict(d_out=P, out_stride=40), INVALID),
    (dict(rank=0), INVALID), (dict(n_in=0), INVALID), (dict(rank=129), UNSUPPORTED), (dict(n_seqs=4097), UNSUPPORTED), (dict(n_in=(1 << 22) + 1), UNSUPPORTED),
    (dict(x_dtype=ans.ANS_F32), UNSUPPORTED), (dict(y_dtype=ans.ANS_E4M3), UNSUPPORTED), (dict(x_stride=1 << 37), UNSUPPORTED),
    (dict(rows=0, d_x=None), 0), (dict(n_out=0, d_b=None), 0), (dict(n_seqs=0, d_which=None), 0)])
def test_adapters(kw, rc):
    assert adapters(**kw) == rc


CACHE = dict(d_k_codes=P, d_k_scales=P, d_v_codes=P, d_v_scales=P, n_pages=4, page_size=16, heads=2, head_dim=64)
BATCH = dict(d_tables=P, table_stride=4, table_pages=4, n_seqs=2, rows=3, d_lengths=P, d_starts=P)
CACHE_CASES = [
    *((dict([(f, None)]), INVALID) for f in ("d_k_codes", "d_k_scales", "d_v_codes", "d_v_scales", "d_tables", "d_lengths", "d_starts", "status")),
    *((dict([(f, P + 8)]), INVALID) for f in ("d_k_codes", "d_k_scales", "d_v_codes", "d_v_scales")), *((dict([(f, P + 2)]), INVALID) for f in ("d_tables", "d_lengths", "d_starts")),
    (dict(table_stride=3), INVALID), (dict(page_size=0), INVALID), (dict(heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(page_size=24), UNSUPPORTED),
    (dict(page_size=272), UNSUPPORTED), (dict(head_dim=72), UNSUPPORTED), (dict(head_dim=272), UNSUPPORTED), (dict(n_seqs=4097), UNSUPPORTED),
    (dict(table_stride=FAR), UNSUPPORTED), (dict(rows=0, d_starts=None), 0), (dict(n_seqs=0, d_tables=None), 0)]


def parts(kw):
    cache, batch, rest = dict(CACHE), dict(BATCH), {}
    for k, v in kw.items():
        (cache if k in cache else batch if k in batch else rest)[k] = v
    return B.ans_block_cache_desc(**cache), B.ans_batch_desc(**batch), rest


def write(status=P, **kw):
    cache, batch, rest = parts(kw)
    a = dict(k=P, v=P, dtype=ans.ANS_BF16, strides=(128, 64, 128, 64)) | rest
    return ans.lib().ans_block_cache_write(cache, batch, a["k"], a["v"], a["dtype"], *a["strides"], status, None)


@pytest.mark.parametrize("kw,rc", CACHE_CASES + [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=P + 1), INVALID), (dict(dtype=ans.ANS_F32, v=P + 2), INVALID), (dict(dtype=ans.ANS_U8), UNSUPPORTED),
    (dict(dtype=ans.ANS_E4M3), UNSUPPORTED), (dict(strides=(FAR, 64, 128, 64)), UNSUPPORTED), (dict(strides=(128, 64, 128, FAR)), UNSUPPORTED)])
def test_block_cache_write(kw, rc):
    assert write(**kw) == rc


def attend(status=P, **kw):
    cache, batch, rest = parts(kw)
    d = B.ans_attend_desc(d_q=P, d_out=2 * P, q_token_stride=256, q_head_stride=64, out_token_stride=256, out_head_stride=64, q_heads=4, causal=1, scale=0.125)
    return ans.lib().ans_attend(cache, batch, changed(d, rest), status, None)


@pytest.mark.parametrize("kw,rc", CACHE_CASES + [
    (dict(d_q=None), INVALID), (dict(d_out=None), INVALID), (dict(d_q=P + 8), INVALID), (dict(d_out=P + 2), INVALID), (dict(q_token_stride=260), INVALID),
    (dict(q_head_stride=68), INVALID), (dict(out_head_stride=65), INVALID), (dict(q_heads=3), INVALID), (dict(q_heads=0), INVALID), (dict(q_heads=258), UNSUPPORTED),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(d_out=P, out_token_stride=512), INVALID),
    (dict(q_token_stride=FAR), UNSUPPORTED), (dict(rows=(1 << 31) - 1), UNSUPPORTED)])
def test_attend(kw, rc):
    assert attend(**kw) == rc


def test_room_is_asked_for_with_the_same_checks():
    out = ctypes.c_size_t()
    cache, batch, _ = parts(dict(head_dim=72))
    assert ans.lib().ans_attend_room_bytes(cache, batch, B.ans_attend_desc(d_q=P, d_out=P, q_heads=4), ctypes.byref(out)) == UNSUPPORTED
    assert ans.lib().ans_attend_room_bytes(None, batch, None, ctypes.byref(out)) == INVALID
    assert ans.lib().ans_adapters_room_bytes(B.ans_adapters_desc(rank=0, n_in=4), ctypes.byref(out)) == INVALID
    assert ans.lib().ans_adapters_room_bytes(B.ans_adapters_desc(rank=8, n_in=4, rows=2, n_seqs=2, n_out=4), ctypes.byref(out)) == 0 and out.value == 0


def test_descriptors_are_those_of_the_header():
    """Sizes as a C compiler lays the header's structures out (LP64)."""
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["ans_pages_desc", "ans_adapters_desc", "ans_block_cache_desc", "ans_batch_desc", "ans_attend_desc"]
    source = '#include <stdio.h>\n#include "ans_b200.h"\nint main(void) {' + "".join(f'printf("%zu\\n", sizeof({n}));' for n in names) + "return 0; }\n"
    with tempfile.TemporaryDirectory() as at:
        with open(os.path.join(at, "s.c"), "w") as f:
            f.write(source)
        subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), "-o", os.path.join(at, "s"), os.path.join(at, "s.c")])
        sizes = [int(v) for v in subprocess.check_output([os.path.join(at, "s")]).split()]
    assert sizes == [ctypes.sizeof(getattr(B, n)) for n in names]
