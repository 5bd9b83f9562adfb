"""What the workspace query of gdn_attention_paged says for sizes that the call refuses (C ABI), and what the binding says to a
cache that is incomplete, CPU."""
import pytest
import torch

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


@pytest.mark.parametrize("missing", ["k_cache", "v_cache", "block_table", "seq_lens"])
@pytest.mark.parametrize("what", [None, 3, [1]])
def test_a_cache_without_one_of_its_tensors(missing, what):
    """Named, with a TypeError, whatever stands in its place."""
    kw = dict(k_cache=torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), v_cache=torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16),
              block_table=torch.zeros(1, 3, dtype=torch.int32), seq_lens=torch.zeros(1, dtype=torch.int32), cu_seqlens=None,
              k_scale=None, v_scale=None)
    kw[missing] = what
    with pytest.raises(TypeError, match=missing):
        gdn._cache_args(-1, *kw.values(), 1, 2, 64)   # (-1: the number that torch gives the CPU)
