"""What the handles and the entry points behind them refuse before they touch a GPU."""
import pytest

import paper_2406_06237_b200 as ans

INVALID, UNSUPPORTED = ans.ANS_ERR_INVALID_ARG, ans.ANS_ERR_UNSUPPORTED
P = 1 << 20                                              # an address on every boundary asked for; never read


@pytest.mark.parametrize("kw,rc", [
    (dict(d_from=None), INVALID), (dict(d_to=None), INVALID), (dict(d_from=P + 1), INVALID), (dict(d_to=P + 8), INVALID),
    (dict(dtype=ans.ANS_F32), UNSUPPORTED), (dict(dtype=ans.ANS_U8), UNSUPPORTED), (dict(rows=(1 << 30) + 1), UNSUPPORTED),
    (dict(k=(1 << 22) + 1), UNSUPPORTED), (dict(stride=1 << 37), UNSUPPORTED), (dict(step=1 << 37), UNSUPPORTED),
    (dict(rows=1 << 30, k=1 << 22), UNSUPPORTED), (dict(rows=0, d_from=None), 0), (dict(k=0, d_to=None), 0)])
def test_product_rows(kw, rc):
    a = {**dict(d_from=P, stride=65, step=1, rows=4, k=65, dtype=ans.ANS_BF16, d_to=P), **kw}
    assert ans.lib().ans_product_rows(*(a[f] for f in ("d_from", "stride", "step", "rows", "k", "dtype", "d_to")), None) == rc
