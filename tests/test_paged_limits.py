"""What the workspace query of gdn_attention_paged says for sizes that the call refuses (C ABI, CPU)."""
import pytest

import paper_2607_14568_amd as gdn
from test_paged_refusals import A, INVALID, UNSUPPORTED, _attention

SIZES = dict(B=1, T=1, H=16, Hkv=8, d=128, page=64, max_pages=500, n=0)


def _need(**kw):
    a = dict(SIZES, **kw)
    return gdn.gdn_attention_paged_workspace_bytes(a["B"], a["T"], a["H"], a["Hkv"], a["d"], a["page"], a["max_pages"], a["n"])


@pytest.mark.parametrize("kw,code", [
    (dict(page=48), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=256), UNSUPPORTED), (dict(page=64, max_pages=(1 << 24) + 1), UNSUPPORTED),
    (dict(page=128, max_pages=2 ** 31 - 1), UNSUPPORTED), (dict(H=1 << 14, Hkv=8), UNSUPPORTED), (dict(T=1 << 26), UNSUPPORTED),
    (dict(B=1 << 13, T=1 << 13), UNSUPPORTED), (dict(T=1 << 26, n=8), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(page=0), INVALID),
    (dict(max_pages=-1), INVALID), (dict(Hkv=32), INVALID), (dict(n=-1), INVALID), (dict(B=2, n=3), INVALID)])
def test_no_workspace_for_what_is_refused(kw, code):
    """0 bytes for every size that the call turns down, and the call's answer beside it."""
    assert _attention(**dict(SIZES, **kw), cu=A if kw.get("n") else None, ws=A, ws_bytes=1 << 40) == code
    assert _need(**kw) == 0


def test_workspace_at_the_limits():
    """The largest sizes that are implemented have one where a sequence may be cut."""
    assert _need() > 0 and _need(page=16) > 0 and _need(page=128, max_pages=1 << 23) > 0 and _need(d=64) > 0
    assert _need(H=1 << 13, Hkv=8) > 0
