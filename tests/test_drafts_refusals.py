"""What the entry points of a drafted step refuse: argument checks of the C ABI (all ahead of the first HIP call) and of the
binding, CPU."""
import pytest
import torch

import paper_2607_14568_amd as gdn
from test_paged_refusals import CACHE, SIZES, _cache_kw

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
A = 1 << 20   # a fake, aligned device address (never dereferenced)


def _tables(**kw):
    a = dict(lens=A, new=A, shared=A, table=A, held=A, free=A, n_free=A, missing=A, cu=A, pos=A, slots=A, n=3, rows=7, page=16,
             n_pages=9, max_pages=4)
    a.update(kw)
    return gdn.lib().gdn_cache_tables(*[a[x] for x in ("lens", "new", "shared", "table", "held", "free", "n_free", "missing", "cu", "pos",
                                                       "slots", "n", "rows", "page", "n_pages", "max_pages")], None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), INVALID), (dict(rows=-1), INVALID), (dict(page=0), INVALID), (dict(page=48), UNSUPPORTED), (dict(n_pages=0), INVALID),
    (dict(max_pages=0), INVALID), (dict(max_pages=1 << 27), UNSUPPORTED), (dict(n=1 << 20, max_pages=1 << 10), UNSUPPORTED), (dict(n_pages=1 << 30), UNSUPPORTED),
    (dict(rows=1 << 30), UNSUPPORTED), (dict(lens=None), INVALID), (dict(table=None), INVALID), (dict(held=None), INVALID),
    (dict(free=None), INVALID), (dict(n_free=None), INVALID), (dict(cu=None), INVALID), (dict(new=None), INVALID),
    (dict(new=None, cu=None, pos=None), INVALID), (dict(lens=A + 2), INVALID), (dict(shared=A + 1), INVALID),
    (dict(missing=A + 2), INVALID), (dict(pos=A + 2), INVALID), (dict(slots=A + 4), INVALID)])
def test_tables_refuse(kw, code):
    assert _tables(**kw) == code
    assert gdn.lib().gdn_last_error_message()


def _shared(**kw):
    a = dict(_cache_kw(), pre=A, cg=None, groups=1, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return gdn.lib().gdn_attention_shared(*[a[x] for x in ("q", "kc", "vc", "ks", "vs", "table", "lens", "pre", "cg", "groups", "qo", "B", "T",
                                                          "H", "Hkv", "d", "page", "n_pages", "max_pages", "cu", "n", "io", "ct", "scale",
                                                          "ws", "ws_bytes")], None)


@pytest.mark.parametrize("kw,code", SIZES + CACHE + [
    (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(qo=A + 8), INVALID), (dict(pre=None), INVALID), (dict(pre=A + 2), INVALID),
    (dict(groups=0), INVALID), (dict(groups=3, cg=A), INVALID), (dict(groups=2), INVALID), (dict(cg=A + 2), INVALID),
    (dict(B=2049), UNSUPPORTED), (dict(T=1 << 28, H=1, Hkv=1), UNSUPPORTED), (dict(cu=A, n=2049, B=1, T=4000), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE),
    (dict(ws=A + 16), INVALID)])
def test_shared_refuses(kw, code):
    assert _shared(**kw) == code


def test_shared_workspace():
    need = gdn.gdn_attention_shared_workspace_bytes
    sizes = (2, 3, 4, 2, 128, 64, 4, 0, 1)
    n = need(*sizes)
    assert n > 0 and n % 256 == 0 and _shared(ws_bytes=n - 1) == WORKSPACE
    for i, bad in enumerate([0, 0, 0, 3, 96, 48, 0, -1, 0]):
        assert need(*(bad if j == i else x for j, x in enumerate(sizes))) == 0, (i, bad)
    assert need(2, 3, 4, 2, 128, 64, 4, 2, 1) == 0 and need(2, 3, 4, 2, 128, 64, 4, 0, 3) == 0 and need(2049, 1, 4, 2, 128, 64, 4) == 0
    assert need(1, 9, 4, 2, 128, 64, 4, 3, 3) > 0


def _draft(**kw):
    a = dict(q=A, k=A, v=A, g=A, beta=A, S=A, o=A, keep=A, B=2, T=3, H=4, Hk=2, dk=128, dv=64, cu=None, n=0, io=gdn.GDN_BF16, scale=1.0,
             flags=0)
    a.update(kw)
    return gdn.lib().gdn_draft_step(*[a[x] for x in ("q", "k", "v", "g", "beta", "S", "o", "keep", "B", "T", "H", "Hk", "dk", "dv", "cu", "n",
                                                     "io", "scale", "flags")], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INVALID), (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(Hk=3), INVALID), (dict(Hk=8), INVALID), (dict(Hk=0), INVALID),
    (dict(dk=96), UNSUPPORTED), (dict(dv=32), UNSUPPORTED), (dict(cu=A), INVALID), (dict(n=2), INVALID), (dict(cu=A, n=-1), INVALID),
    (dict(cu=A, n=2), INVALID), (dict(cu=A + 2, n=2, B=1), INVALID), (dict(io=2), INVALID), (dict(flags=4), INVALID),
    (dict(flags=gdn.GDN_PLAN_WIDE), INVALID), (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(g=None), INVALID), (dict(beta=None), INVALID), (dict(S=None), INVALID), (dict(S=A + 8), INVALID),
    (dict(k=A + 1), INVALID), (dict(keep=A + 2), INVALID), (dict(g=A + 2), INVALID), (dict(B=1 << 22, T=1, H=16), UNSUPPORTED),
    (dict(T=1 << 29), UNSUPPORTED)])
def test_draft_refuses(kw, code):
    assert _draft(**kw) == code


def _verify(**kw):
    a = dict(p=A, q=A, drafts=A, lens=A, u=A, tokens=A, counts=A, n=3, m=2, V=100, ps=100, qs=100, dt=gdn.GDN_F32, ws=A, ws_bytes=1 << 20)
    a.update(kw)
    return gdn.lib().gdn_draft_verify(*[a[x] for x in ("p", "q", "drafts", "lens", "u", "tokens", "counts", "n", "m", "V", "ps", "qs", "dt",
                                                       "ws", "ws_bytes")], None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), INVALID), (dict(m=-1), INVALID), (dict(V=0), INVALID), (dict(V=1 << 30, ps=1 << 30, qs=1 << 30), UNSUPPORTED),
    (dict(m=1 << 20), UNSUPPORTED), (dict(n=1 << 29), UNSUPPORTED), (dict(p=None), INVALID), (dict(u=None), INVALID),
    (dict(tokens=None), INVALID), (dict(counts=None), INVALID), (dict(drafts=None), INVALID), (dict(m=0), INVALID),
    (dict(m=0, drafts=None), INVALID), (dict(m=0, drafts=None, q=None), INVALID), (dict(ps=99), INVALID), (dict(qs=99), INVALID),
    (dict(dt=2), INVALID), (dict(p=A + 2), INVALID), (dict(q=A + 1, dt=gdn.GDN_BF16), INVALID), (dict(u=A + 2), INVALID),
    (dict(tokens=A + 2), INVALID), (dict(ws=None), WORKSPACE), (dict(ws_bytes=10), WORKSPACE), (dict(ws=A + 16), INVALID)])
def test_verify_refuses(kw, code):
    assert _verify(**kw) == code


def test_verify_workspace():
    need = gdn.gdn_draft_verify_workspace_bytes
    assert need(3, 2, 100) > 0 and need(64, 0, 131072) >= need(64, 5, 100) and need(0, 2, 100) == need(3, -1, 100) == need(3, 2, 0) == 0


def test_nothing_to_do():
    assert _shared(T=0, q=None) == 0 and _draft(T=0, k=None) == 0


def test_binding_refuses():
    x, i = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        gdn.gdn_cache_tables(i, i[None], i, i, i, 16)
    with pytest.raises(TypeError):
        gdn.gdn_attention_shared(x, x, x, i[None], i, i)
    with pytest.raises(TypeError):
        gdn.gdn_draft_step(x, x, x, x, x, x)
    with pytest.raises(TypeError):
        gdn.gdn_draft_step(None, x.half(), x, x, x, x)
    with pytest.raises(TypeError):
        gdn.gdn_draft_verify(torch.zeros(1, 2, 5), torch.zeros(1, 2))


def test_rows_of_wider_probabilities():
    """The distance between rows that the binding passes on, and the layouts that it refuses."""
    class Cuda(torch.Tensor):
        is_cuda = True

    def step(t, shape=None):
        return gdn._probabilities(t.as_subclass(Cuda), "p", shape)[1]
    wide = torch.zeros(3, 4, 50)
    assert step(wide) == 50 and step(wide[..., :40]) == 50 and step(wide[:, :1]) == 200 and step(wide[:1, 1:2, :40]) == 40
    for bad in (wide[:, :3], wide.transpose(0, 1), wide[..., ::2], wide[0]):
        with pytest.raises(ValueError):
            step(bad)
    with pytest.raises(ValueError):
        step(wide, (3, 3, 50))
    with pytest.raises(TypeError):
        step(wide.half())
