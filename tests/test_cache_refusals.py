"""What dd_qk_norm_rope, dd_cache_append and dd_cached_attention refuse, through the C ABI and through the binding (no GPU work), and
the plain forms that their results are compared with."""
import ctypes

import numpy as np
import pytest
import torch

from tests import _cache_reference as ref

INVALID, UNSUPPORTED = -1, -2


@pytest.fixture(scope="module")
def dd():
    from paper_2604_05250_b200 import binding, build
    build.build()
    return binding


def P(x=64):
    return ctypes.c_void_p(x)                  # never dereferenced: validation comes first


def strides(dd, batch=1024, token=256, head=128):
    return ctypes.byref(dd._Strides(batch, token, head))


def rotation(dd, cos=64, sin=64, positions=8, dims=64, interleaved=0):
    return ctypes.byref(dd._Rotation(cos, sin, positions, dims, interleaved))


def cache(dd, k=64, v=64, ks=64, vs=64, table=64, num_pages=4, max_pages=4, page=16, heads=2, D=128):
    return ctypes.byref(dd._Cache(k, v, ks, vs, table, num_pages, max_pages, page, heads, D))


def test_norm_rope(dd):
    L = dd.lib()

    def call(q=P(), qs=None, H=2, k=P(), ks=None, Hkv=1, wq=P(), wk=P(), eps=1e-6, rot=None, out_q=P(), out_k=P(), B=1, N=4, D=128, layout=1):
        return L.dd_qk_norm_rope(q, qs or strides(dd), H, k, ks or strides(dd), Hkv, wq, wk, eps, rot, None, out_q, out_k, B, N, D, layout, None)
    assert call(q=None) == call(out_q=None) == call(k=None) == call(out_k=None) == INVALID
    assert L.dd_qk_norm_rope(P(), None, 2, None, None, 0, None, None, 1e-6, None, None, P(), None, 1, 4, 128, 1, None) == INVALID
    assert call(H=0) == call(Hkv=-1) == call(B=0) == call(N=0) == call(D=0) == call(layout=2) == INVALID
    assert call(eps=-1e-6) == call(eps=float("nan")) == call(eps=float("inf")) == INVALID
    assert call(qs=strides(dd, token=-256)) == INVALID
    assert call(D=96) == call(q=P(72)) == call(wq=P(66)) == call(wk=P(66)) == call(out_q=P(72)) == call(out_k=P(72)) == UNSUPPORTED
    assert call(qs=strides(dd, head=132)) == call(ks=strides(dd, batch=4)) == UNSUPPORTED
    assert call(rot=rotation(dd, dims=24)) == call(rot=rotation(dd, dims=144)) == call(rot=rotation(dd, cos=72)) == UNSUPPORTED
    assert call(rot=rotation(dd, cos=0)) == call(rot=rotation(dd, sin=0)) == call(rot=rotation(dd, positions=0)) == INVALID
    assert call(rot=rotation(dd, dims=-16)) == INVALID
    assert call(B=2 ** 20, N=2 ** 20) == UNSUPPORTED


def test_cache_append(dd):
    L = dd.lib()

    def call(k=P(), ks=None, v=P(), vs=None, c=None, start=P(), w=None, eps=1e-6, rot=None, B=1, N=4):
        return L.dd_cache_append(k, ks or strides(dd), v, vs or strides(dd), c or cache(dd), start, None, None, w, eps, rot, B, N, None)
    assert call(k=None) == call(v=None) == call(start=None) == call(B=0) == call(N=-1) == call(eps=float("nan")) == INVALID
    for bad in ("k", "v", "ks", "vs", "table"):
        assert call(c=cache(dd, **{bad: 0})) == INVALID
    for bad in ("num_pages", "max_pages", "page", "heads", "D"):
        assert call(c=cache(dd, **{bad: 0})) == INVALID
    assert call(c=cache(dd, page=48)) == call(c=cache(dd, page=256)) == call(c=cache(dd, D=256)) == call(c=cache(dd, k=72)) == UNSUPPORTED
    assert call(c=cache(dd, num_pages=2 ** 26)) == call(c=cache(dd, max_pages=2 ** 27)) == call(c=cache(dd, ks=66)) == UNSUPPORTED
    assert call(vs=strides(dd, token=12)) == call(v=P(68)) == call(w=P(72)) == call(rot=rotation(dd, dims=8)) == UNSUPPORTED
    assert call(ks=strides(dd, head=-8)) == INVALID
    # 2 (keys and values) * heads * sequences * pages that tokens fall into
    assert call(B=2 ** 29) == UNSUPPORTED


def test_cached_attention(dd):
    L = dd.lib()

    def call(q=P(), qs=None, c=None, lens=P(), out=P(), os=None, B=1, H=4, Nq=1, scale=0.1, ws=P(), size=1 << 30):
        return L.dd_cached_attention(q, qs or strides(dd), c or cache(dd), lens, out, os or strides(dd), B, H, Nq, scale, ws, size, None)
    assert call(q=None) == call(lens=None) == call(out=None) == call(ws=None) == call(B=0) == call(H=0) == call(Nq=0) == INVALID
    assert call(H=5) == call(scale=float("nan")) == call(scale=float("inf")) == call(c=cache(dd, table=0)) == INVALID
    assert call(scale=-1.0) == call(ws=P(72)) == call(q=P(72)) == call(out=P(72)) == call(os=strides(dd, head=4)) == UNSUPPORTED
    assert call(Nq=2 ** 30) == call(B=2 ** 30, Nq=8) == call(c=cache(dd, page=8)) == UNSUPPORTED
    assert call(qs=strides(dd, batch=-8)) == INVALID
    assert L.dd_cached_attention_workspace_bytes(0, 4, 1, cache(dd)) == L.dd_cached_attention_workspace_bytes(1, 5, 1, cache(dd)) == 0
    assert L.dd_cached_attention_workspace_bytes(1, 4, 1, None) == 0


def test_binding_words_what_it_refuses(dd):
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        dd.qk_norm_rope(q)
    with pytest.raises(ValueError, match="contiguous rows"):
        dd.qk_norm_rope(q.float())
    with pytest.raises(ValueError, match="contiguous rows"):
        dd.qk_norm_rope(q.transpose(2, 3))
    with pytest.raises(ValueError, match="layout"):
        dd.qk_norm_rope(q, layout="nbhd")
    with pytest.raises(ValueError, match="layout"):
        dd.cached_attention(q, None, None, None, layout="nbhd")
    c = dd.new_cache(3, 2, 16, 64, device="cpu")
    assert c.k.dtype == torch.float8_e4m3fn and c.k.shape == (3, 2, 16, 64) and c.v_scale.shape == (3, 2)
    table = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="cache.k: expected a device tensor"):
        dd.cache_append(q, q, c, table, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="cache.v"):
        dd.cached_attention(q, c._replace(k=_on_device(c.k), v=c.v.float()), table, None)


def test_binding_takes_a_tuple_as_a_cache_and_nothing_else(dd):
    """Four tensors in a plain tuple are a cache, as for the native host side; other things are refused in words."""
    q, table, start = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    c = tuple(dd.new_cache(3, 2, 16, 64, device="cpu"))
    with pytest.raises(ValueError, match="cache.k: expected a device tensor"):
        dd.cache_append(q, q, c, table, start)
    with pytest.raises(ValueError, match="cache.k: expected a device tensor"):
        dd.cached_attention(q, c, table, start)
    for bad in (None, c[:3], list(c), 7):
        with pytest.raises(TypeError, match="cache: expected a Cache"):
            dd.cache_append(q, q, bad, table, start)
        with pytest.raises(TypeError, match="cache: expected a Cache"):
            dd.cached_attention(q, bad, table, start)
    with pytest.raises(TypeError, match="cache.k: expected a torch.Tensor"):
        dd.cached_attention(q, (None, *c[1:]), table, start)
    with pytest.raises(ValueError, match="cache.k: expected"):
        dd.cached_attention(q, (c[0][0], *c[1:]), table, start)


class _on_device(torch.Tensor):
    """A host tensor that says it is on the device: gets past the first check, to the next one."""

    @staticmethod
    def __new__(cls, t):
        return torch.Tensor._make_subclass(cls, t)

    is_cuda = True


def test_e4m3_rounding_of_the_plain_form():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    finite = every[~every.isnan()].unique()
    assert np.array_equal(ref.to_e4m3(finite.double().numpy()), finite.double().numpy())
    # between neighbours: the nearer one, and the one of even mantissa in the middle
    x = torch.cat([finite[:-1] + f * (finite[1:] - finite[:-1]) for f in (0.25, 0.5, 0.75)])
    assert np.array_equal(ref.to_e4m3(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())
    assert ref.to_e4m3(1e9) == 448 and ref.to_e4m3(-460.0) == -448 and np.isnan(ref.to_e4m3(np.nan))


def test_scale_exponents_of_the_plain_form():
    assert [ref.exponent(x) for x in (448.0, 448.1, 896.0, 224.0, 0.0, 1e30)] == [0, 1, 1, -1, -60, 60]


def test_plain_attention_is_an_average_of_values():
    g = np.random.default_rng(0)
    pools = [g.normal(size=(4, 1, 16, 64)), np.full((4, 1, 16, 64), 3.0)]
    scales = [np.ones((4, 1)), np.full((4, 1), 0.5)]
    out, bar = ref.attention(g.normal(size=(1, 2, 2, 64)), pools, scales, np.array([[2, -1, 0]]), [40], 0.125)
    assert np.allclose(out, 1.5) and (bar > 0).all()
    out, _ = ref.attention(g.normal(size=(1, 2, 2, 64)), pools, scales, np.array([[-1, -1, 0]]), [32], 0.125)
    assert not out.any()


def test_plain_rotation_keeps_lengths_and_angles():
    g = np.random.default_rng(1)
    a = np.arange(20)[:, None] * 10.0 ** (-np.arange(8) / 8)[None]
    q, k = g.normal(size=(1, 1, 64)), g.normal(size=(1, 1, 64))
    for interleaved in (False, True):
        turned = lambda x, p: ref.norm_rotate(x, None, 0, np.cos(a), np.sin(a), [p], interleaved)[0, 0]  # noqa: E731
        assert np.isclose(np.linalg.norm(turned(q, 7)), np.linalg.norm(q))
        # the product goes by the distance alone
        assert np.isclose(turned(q, 9) @ turned(k, 4), turned(q, 17) @ turned(k, 12))
