"""dd_cached_attention: which scales of pages it may look at, and the range of those that it does."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cached_attention import check, dd, make  # noqa: F401  (dd: the fixture)

pytestmark = pytest.mark.gpu


def reserve(s, page, how, scale):
    """Valid entries in the table behind every sequence's last page: pages of their own, whose bytes are NaN and whose scales are
    `scale`, or page 0 (padding), which gets such scales where it holds nobody's tokens."""
    table, total = s["table_np"].copy(), s["cache"][0].shape[0]
    used = {int(p) for b, n in enumerate(s["lens_np"]) for p in table[b, :-(-n // page)]}
    behind = [(b, p) for b, n in enumerate(s["lens_np"]) for p in range(-(-n // page), table.shape[1])]
    spare = [p for p in range(total) if p not in used]
    for i, (b, p) in enumerate(behind):
        table[b, p] = spare[i % len(spare)] if how == "spare" else 0
    cache = [c.clone() for c in s["cache"]]
    for p in spare:
        for c in cache[2:]:
            c[p] = scale
    return tuple(cache), torch.from_numpy(table).cuda()


@pytest.mark.parametrize("Nq", [1, 20, 40])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("how", ["spare", "padded"])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** 24, 2.0 ** 60, float("inf"), float("nan")])
def test_pages_behind_the_end_are_not_looked_at(dd, Nq, page, how, scale):  # noqa: F811
    """Pages given out ahead, and padding: bit for bit what a table without them gives, whatever stands in them."""
    s = make(Nq + page, [1, 15, 17, 40, 65, 100, 129, 300, 0], 2, 2 if Nq == 1 else 1, Nq, 128 if page < 64 else 64, page, extra_pages=8)
    want = check(dd, s)
    cache, table = reserve(s, page, how, scale)
    got = dd.cached_attention(s["q"], dd.Cache(*cache), table, s["lens"])
    assert torch.equal(got, want)


@pytest.mark.parametrize("Nq", [1, 40])
def test_a_page_that_held_infinity_and_is_reserved(dd, Nq):  # noqa: F811
    """An append of an infinite value leaves a scale of 2^60; its page, given to another sequence for later, changes nothing there."""
    heads, D, page = 2, 128, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = dd.new_cache(4, heads, page, D)
    as_int = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v = (torch.randn(1, 50, heads, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(1, Nq, heads, D, generator=g, device="cuda").bfloat16()
    dd.cache_append(k, v, cache, as_int(0, 1).view(1, 2), as_int(0))
    want = dd.cached_attention(q, cache, as_int(0, 1, -1).view(1, 3), as_int(50))
    bad = v[:, :1].clone()
    bad[..., 0] = float("inf")
    dd.cache_append(k[:, :1], bad, cache, as_int(2).view(1, 1), as_int(0))
    assert float(cache.v_scale[2, 0]) == 2.0 ** 60
    got = dd.cached_attention(q, cache, as_int(0, 1, 2).view(1, 3), as_int(50))
    assert want.abs().max() > 0.1 and torch.equal(got, want)


@pytest.mark.parametrize("Nq", [1, 20, 40])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_values_of_zero_scale_behind_missing_pages(dd, Nq, page):  # noqa: F811
    """The first tile's pages are not there, the next one's values stand under scales of zero: its keys count all the same, whether a
    positive scale follows (in the same share or in another) or not."""
    lens, heads = [500, 256, 390, 300] * 12, 8
    per = 128 // page
    s = make(page + Nq, lens, heads, 1, Nq, 64, page, strength=0.01, missing=[(b, p) for b in range(len(lens)) for p in range(per)])
    for b in range(len(lens)):
        for p in range(per, 2 * per):
            s["scales"][1][s["table_np"][b, p]] = 0.0
            s["cache"][3][s["table_np"][b, p]] = 0.0
    check(dd, s)


@pytest.mark.parametrize("Nq", [1, 20, 40])
@pytest.mark.parametrize("low,high", [(-100, -96), (-60, -40), (40, 60), (70, 76), (-100, 76)])
def test_range_of_scales(dd, Nq, low, high):  # noqa: F811
    """Values under very small and very large scales (numbers below 2^100 / kv_len), and keys under as small ones."""
    s = make(Nq + high + 100, [300, 70], 2, 2, Nq, 128, 16)
    g = np.random.default_rng(low + high + 200)
    s["scales"][1][:] = 2.0 ** g.integers(low, high + 1, size=s["scales"][1].shape)
    s["cache"][3][:] = torch.from_numpy(s["scales"][1]).float().cuda()
    if high < 0:
        s["scales"][0][:] = 2.0 ** g.integers(low, high + 1, size=s["scales"][0].shape)
        s["cache"][2][:] = torch.from_numpy(s["scales"][0]).float().cuda()
    check(dd, s)


@pytest.mark.parametrize("Nq", [1, 40])
def test_values_of_zero_under_the_largest_scale(dd, Nq):  # noqa: F811
    s = make(Nq, [300], 2, 1, Nq, 128, 64)
    page = int(s["table_np"][0, 1])
    s["pools"][1][page] = 0.0
    s["cache"][1].view(torch.uint8)[page] = 0
    s["scales"][1][page] = 2.0 ** 100
    s["cache"][3][page] = 2.0 ** 100
    got = dd.cached_attention(s["q"], dd.Cache(*s["cache"]), s["table"], s["lens"])
    assert got.isfinite().all()


@pytest.mark.parametrize("Nq", [1, 20, 40])
@pytest.mark.parametrize("by", [-93, -50, 50, 93])
def test_scales_times_a_power_of_two(dd, Nq, by):  # noqa: F811
    """The same bits under another exponent, from 2^-100 to 2^100."""
    s = make(Nq, [300, 70, 1], 2, 2, Nq, 128, 32)          # scales of 2^-11 to 2^-5
    s["cache"][3].mul_(2.0 ** 4)                             # 2^-7 to 2^-1
    if by > 0:
        s["cache"][3].mul_(2.0 ** 8)                         # 2 to 2^7
    cache = dd.Cache(*s["cache"])
    want = dd.cached_attention(s["q"], cache, s["table"], s["lens"])
    got = dd.cached_attention(s["q"], cache._replace(v_scale=cache.v_scale * 2.0 ** by), s["table"], s["lens"])
    assert torch.equal(got.double(), want.double() * 2.0 ** by)


def test_rows_that_are_not_finite_behind_missing_pages(dd):  # noqa: F811
    """A row of NaN scores never gets a reference point; the rows beside it are the same as without it."""
    s = make(31, [600, 300], 2, 1, 20, 128, 64, missing=[(0, 0), (0, 1), (1, 2)])
    want = check(dd, s)
    s["q"][:, 7, 1] = float("nan")
    got = dd.cached_attention(s["q"], dd.Cache(*s["cache"]), s["table"], s["lens"])
    assert got[:, 7, 1].isnan().all()
    got[:, 7, 1] = want[:, 7, 1]
    assert torch.equal(got, want)
