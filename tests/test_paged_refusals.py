"""What the paged cache's entry points refuse: argument checks of the C ABI (all ahead of the first HIP call) and of the
binding, CPU."""
import ctypes

import pytest
import torch

import paper_2607_14568_amd as gdn

INVALID, UNSUPPORTED = 1, 2
A = 1 << 20   # a fake, aligned device address (never dereferenced)


def _norm(**kw):
    a = dict(q=A, k=A, qo=A, ko=A, B=1, T=4, H=4, Hkv=2, d=128, qs=512, ks=256, qw=A, kw=A, eps=1e-6, f=A, rot=128, pos=None,
             cu=None, n=0, io=gdn.GDN_BF16, flags=0)
    a.update(kw)
    return gdn.lib().gdn_qk_norm_rope(a["q"], a["k"], a["qo"], a["ko"], a["B"], a["T"], a["H"], a["Hkv"], a["d"], a["qs"], a["ks"],
                                      a["qw"], a["kw"], a["eps"], a["f"], a["rot"], a["pos"], a["cu"], a["n"], a["io"], a["flags"], None)


SIZES = [(dict(B=0), INVALID), (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(Hkv=3), INVALID), (dict(Hkv=8), INVALID),
         (dict(Hkv=0), INVALID), (dict(d=0), INVALID), (dict(d=96), UNSUPPORTED), (dict(cu=A), INVALID), (dict(n=2), INVALID),
         (dict(cu=A, n=-1), INVALID), (dict(cu=A, n=2, B=2), INVALID), (dict(cu=A + 2, n=2), INVALID), (dict(io=2), INVALID),
         (dict(io=7), INVALID), (dict(H=1 << 14, Hkv=1 << 14), UNSUPPORTED), (dict(T=1 << 29), UNSUPPORTED)]
TURN = [(dict(flags=1), INVALID), (dict(flags=1024), INVALID), (dict(rot=0), INVALID), (dict(f=None), INVALID), (dict(rot=-16), INVALID),
        (dict(rot=144), INVALID), (dict(rot=24), UNSUPPORTED), (dict(f=A + 4), INVALID), (dict(eps=-1.0), INVALID),
        (dict(eps=float("nan")), INVALID), (dict(kw=A + 2), INVALID)]


@pytest.mark.parametrize("kw,code", SIZES + TURN + [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(qo=None), INVALID), (dict(ko=None), INVALID), (dict(q=A + 8), INVALID),
    (dict(ko=A + 8), INVALID), (dict(qs=504), INVALID), (dict(qs=516), INVALID), (dict(ks=0), INVALID), (dict(pos=A + 2), INVALID)])
def test_norm_rope_refuses(kw, code):
    assert _norm(**kw) == code
    assert gdn.lib().gdn_last_error_message()


def _cache_kw(**kw):
    a = dict(q=A, k=A, v=A, qo=A, kc=A, vc=A, ks=None, vs=None, table=A, lens=A, B=2, T=3, H=4, Hkv=2, d=128, page=64, n_pages=9,
             max_pages=4, qs=512, kst=256, vst=256, qw=A, kw=A, eps=1e-6, f=A, rot=64, cu=None, n=0, io=gdn.GDN_BF16,
             ct=gdn.GDN_BF16, flags=0, scale=0.1, ws=None, ws_bytes=0)
    a.update(kw)
    return a


def _append(**kw):
    a = _cache_kw(**kw)
    return gdn.lib().gdn_kv_append(*[a[x] for x in ("q", "k", "v", "qo", "kc", "vc", "ks", "vs", "table", "lens", "B", "T", "H", "Hkv", "d",
                                                    "page", "n_pages", "max_pages", "qs", "kst", "vst", "qw", "kw", "eps", "f", "rot",
                                                    "cu", "n", "io", "ct", "flags")], None)


def _attention(**kw):
    a = _cache_kw(**kw)
    return gdn.lib().gdn_attention_paged(*[a[x] for x in ("q", "kc", "vc", "ks", "vs", "table", "lens", "qo", "B", "T", "H", "Hkv", "d", "page",
                                                         "n_pages", "max_pages", "cu", "n", "io", "ct", "scale", "ws", "ws_bytes")], None)


CACHE = [(dict(ct=0), INVALID), (dict(ct=3), INVALID), (dict(page=0), INVALID), (dict(page=48), UNSUPPORTED), (dict(page=256), UNSUPPORTED),
         (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=1 << 26, page=64), UNSUPPORTED), (dict(kc=None), INVALID),
         (dict(vc=A + 8), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(table=A + 2), INVALID),
         (dict(ks=A), INVALID), (dict(ks=A, vs=A), INVALID), (dict(ct=2), INVALID), (dict(ct=2, ks=A), INVALID),
         (dict(ct=2, ks=A, vs=A + 1), INVALID), (dict(io=gdn.GDN_F32), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", SIZES + TURN[:-1] + CACHE + [
    (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(v=A + 4), INVALID),
    (dict(kst=128), INVALID), (dict(vst=260), INVALID), (dict(qo=A + 8), INVALID)])
def test_append_refuses(kw, code):
    assert _append(**kw) == code


@pytest.mark.parametrize("kw,code", SIZES + CACHE + [(dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(qo=A + 8), INVALID)])
def test_attention_refuses(kw, code):
    assert _attention(**kw) == code


def test_workspace():
    """Needed where a sequence may be cut, never for arguments that are refused; missing, small and misaligned ones."""
    need = gdn.gdn_attention_paged_workspace_bytes
    sizes = dict(B=1, T=1, H=16, Hkv=8, max_pages=500)
    n = need(1, 1, 16, 8, 128, 64, 500)
    assert n > 0 and need(1, 1, 16, 8, 128, 64, 1) == 0 and need(4096, 1, 16, 8, 128, 64, 500) == 0
    assert need(1, 64, 16, 8, 128, 64, 500, 8) > 0 and need(1, 2048, 16, 8, 128, 64, 500) > 0
    for bad in [(0, 1, 16, 8, 128, 64, 500), (1, 1, 16, 3, 128, 64, 500), (1, 1, 16, 8, 96, 64, 500), (1, 1, 16, 8, 128, 0, 500),
                (2, 1, 16, 8, 128, 64, 500, 2), (1, 1, 16, 8, 128, 64, 0), (1, 0, 16, 8, 128, 64, 500)]:
        assert need(*bad) == 0, bad
    assert _attention(**sizes) == 3 and _attention(**sizes, ws=A, ws_bytes=n - 1) == 3
    assert _attention(**sizes, ws=A + 16, ws_bytes=n) == INVALID


def test_nothing_to_do():
    assert _norm(T=0, q=None, qo=None) == 0 and _append(T=0, k=None) == 0 and _attention(T=0, q=None) == 0


def test_binding_refuses():
    x = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        gdn.gdn_qk_norm_rope(x, x)
    with pytest.raises(TypeError):
        gdn.gdn_qk_norm_rope(x.half(), x.half())
    with pytest.raises(TypeError):
        gdn.gdn_kv_append(x, x, x, x, i[None], i)
    with pytest.raises(TypeError):
        gdn.gdn_attention_paged(x, x, x, i[None], i)


def test_rows_of_a_projection():
    """The distance between tokens that the binding passes on, and the layouts that it refuses."""
    class Cuda(torch.Tensor):
        is_cuda = True

    def rows(t):
        return gdn._rows(t.as_subclass(Cuda), "q", torch.float32)[1]
    wide = torch.zeros(2, 3, 10, 64)
    assert rows(wide) == 640 and rows(wide[:, :, 2:6]) == 640 and rows(wide[:1, :, 2:6]) == 640 and rows(wide[:, :1, 2:6]) == 1920
    assert rows(wide[:1, :1, 2:6]) == 256
    for bad in (wide[:, :2, 2:6], wide.transpose(1, 2), wide[..., ::2], wide[:, :, ::2], wide[0]):
        with pytest.raises(ValueError):
            rows(bad)
