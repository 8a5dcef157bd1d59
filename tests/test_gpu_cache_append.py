"""dd_qk_norm_rope and dd_cache_append against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from tests import _cache_reference as ref

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def dd():
    from paper_2604_05250_b200 import binding, build
    build.build()
    return binding


def angles(positions, dims):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, dims, 2) / dims)[None]
    return torch.from_numpy(np.cos(a)).float(), torch.from_numpy(np.sin(a)).float()


def rows(g, *shape, spread=0):
    return torch.from_numpy(g.normal(size=shape) * 2.0 ** g.integers(-spread, spread + 1, size=shape[:-1] + (1,))).bfloat16()


def weight_of(g, D):
    return torch.from_numpy(1 + 0.3 * g.normal(size=D)).bfloat16()


def between(got, low, high, what):
    assert np.array_equal(np.isnan(got), np.isnan(low)), f"{what}: NaN at other places"
    ok = np.isnan(low) | ((got >= np.minimum(low, high)) & (got <= np.maximum(low, high)))
    assert ok.all(), f"{what}: {(~ok).sum()} of {ok.size} off, first at {np.argwhere(~ok)[0].tolist()}: {got[~ok][0]} not in {low[~ok][0]}, {high[~ok][0]}"


# ------------------------------------------------------------------------------- norms and rotation

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dims", [0, 16, 48, 64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["bnhd", "bhnd"])
@pytest.mark.parametrize("normed", [(True, True), (False, True), (False, False)])
def test_norm_rope(dd, D, dims, interleaved, layout, normed):
    if dims > D:
        dims = D
    g = np.random.default_rng(D + dims)
    B, N, H, Hkv = 3, 7, 5, 2
    q, k = rows(g, B, N, H, D, spread=4), rows(g, B, N, Hkv, D, spread=4)
    wq, wk = (weight_of(g, D) if n else None for n in normed)
    cos, sin = angles(64, dims) if dims else (None, None)
    start = torch.tensor([0, 57, 20], dtype=torch.int32)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    got = dd.qk_norm_rope(q.cuda(), k.cuda(), q_weight=dev(wq), k_weight=dev(wk), eps=EPS, cos=dev(cos), sin=dev(sin), start=start.cuda(),
                          interleaved=interleaved, layout=layout)
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        y = y.double().cpu().numpy()
        if layout == "bhnd":
            y = y.transpose(0, 2, 1, 3)
        for b in range(B):
            c, s = (None, None) if cos is None else (cos.double().numpy(), sin.double().numpy())
            w64 = None if w is None else w.double().numpy()
            x64 = x[b].double().numpy()
            want = ref.norm_rotate(x64, w64, EPS, c, s, int(start[b]) + np.arange(N), interleaved)
            d = ref.slack(x64, w64, EPS, c)
            between(y[b], ref.to_bf16(want - d), ref.to_bf16(want + d), f"sequence {b}")


def test_norm_rope_queries_alone_views_in_place(dd):
    g = np.random.default_rng(1)
    B, N, H, D = 2, 5, 3, 128
    mixed = rows(g, B, N, (H + 2) * D).cuda()
    q = mixed[..., :H * D].view(B, N, H, D)
    w = weight_of(g, D).cuda()
    cos, sin = (t.cuda() for t in angles(32, D))
    plain = dd.qk_norm_rope(q.contiguous(), q_weight=w, cos=cos, sin=sin)
    assert plain[1] is None
    assert torch.equal(plain[0], dd.qk_norm_rope(q, q_weight=w, cos=cos, sin=sin)[0])
    own = q.contiguous()
    dd.qk_norm_rope(own, q_weight=w, cos=cos, sin=sin, out_q=own)
    assert torch.equal(plain[0], own)
    one = q[:, :1].expand(B, N, H, D)                      # the same row at every position: a stride of zero
    assert torch.equal(dd.qk_norm_rope(one, cos=cos, sin=sin)[0], dd.qk_norm_rope(one.contiguous(), cos=cos, sin=sin)[0])


def test_norm_rope_positions_without_angle(dd):
    g = np.random.default_rng(2)
    q = rows(g, 3, 4, 2, 64).cuda()
    cos, sin = (t.cuda() for t in angles(8, 32))
    start = torch.tensor([-2, 6, 2 ** 31 - 2], dtype=torch.int32, device="cuda")
    out = dd.qk_norm_rope(q, cos=cos, sin=sin, start=start)[0]
    lost = out.isnan().all(-1).all(-1).cpu().numpy()        # never: entries behind `dims` have no angle
    assert not lost.any()
    lost = out[..., :32].isnan().all(-1).all(-1).cpu().numpy()
    assert lost.tolist() == [[True, True, False, False], [False, False, True, True], [True, True, True, True]]
    assert torch.equal(out[..., 32:], q[..., 32:])


def test_norm_rope_zero_rows_and_nan(dd):
    q = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16, device="cuda")
    q[0, 1, 1, 3] = float("nan")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = dd.qk_norm_rope(q, q_weight=w)[0]
    assert not out[0, 0].any() and not out[0, 1, 0].any() and out[0, 1, 1].isnan().all()


# ------------------------------------------------------------------------------- append

def state(seed, B, heads, page, D, width, total=None):
    g = np.random.default_rng(seed)
    total = total or B * width + 2
    table = g.permutation(total)[:B * width].reshape(B, width).astype(np.int32)
    raw = []
    for _ in range(2):
        bits = g.integers(0, 256, size=(total, heads, page, D)).astype(np.uint8)            # every pattern, NaN among them
        raw.append((torch.from_numpy(bits).view(torch.float8_e4m3fn), torch.from_numpy(2.0 ** g.integers(-12, -2, size=(total, heads))).float()))
    return table, raw


def run_append(dd, raw, table, k, v, start, count=None, kv_len=None, w=None, cos=None, sin=None, interleaved=False, exact=None):
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    as_int = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    cache = dd.Cache(raw[0][0].cuda(), raw[1][0].cuda(), raw[0][1].cuda(), raw[1][1].cuda())
    got = dd.cache_append(dev(k), dev(v), cache, torch.from_numpy(table).cuda(), as_int(start), count=as_int(count), kv_len=as_int(kv_len),
                          k_weight=dev(w), eps=EPS, cos=dev(cos), sin=dev(sin), interleaved=interleaved)
    assert got is cache
    torch.cuda.synchronize()
    f64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    pools, scales = [f64(raw[i][0].float()) for i in (0, 1)], [f64(raw[i][1]) for i in (0, 1)]
    want = ref.append(f64(k), f64(v), pools, scales, table, start, count, kv_len, f64(w), EPS, f64(cos), f64(sin), interleaved)
    for i, (x, name) in enumerate(((cache.k, "keys"), (cache.k_scale, "scales of keys"), (cache.v, "values"), (cache.v_scale, "scales of values"))):
        between(x.float().double().cpu().numpy(), *want[i], name)
    # what no token stands at keeps its bytes, not only its numbers
    return cache


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("N,start", [(1, [0, 5, 40]), (3, [0, 15, 30]), (40, [0, 7, 33]), (130, [0, 1, 100])])
@pytest.mark.parametrize("normed", [False, True])
def test_append(dd, D, page, N, start, normed):
    g = np.random.default_rng(N + page)
    width = (max(start) + N + page - 1) // page
    table, raw = state(N * page + D, 3, 2, page, D, width)
    cos, sin = angles(256, D)
    run_append(dd, raw, table, rows(g, 3, N, 2, D, spread=3), rows(g, 3, N, 2, D, spread=3), start, w=weight_of(g, D) if normed else None,
               cos=cos, sin=sin)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("interleaved,dims", [(True, 128), (True, 32), (False, 96), (False, 0)])
def test_append_amid_held_tokens(dd, page, interleaved, dims):
    """A block in the middle computed anew: what was held before and behind it stays, whatever becomes of the pages' scales."""
    g = np.random.default_rng(page + dims)
    B, N, D = 4, 20, 128
    table, raw = state(3, B, 2, page, D, 160 // page)
    cos, sin = angles(200, dims) if dims else (None, None)
    run_append(dd, raw, table, rows(g, B, N, 2, D, spread=6), rows(g, B, N, 2, D, spread=6), [10, 60, 0, 100], kv_len=[130, 70, 15, 90],
               count=[20, 13, 20, 0], cos=cos, sin=sin, interleaved=interleaved)


def test_append_counts_and_places_that_are_not_there(dd):
    g = np.random.default_rng(4)
    B, N, D, page = 6, 33, 64, 16
    table, raw = state(5, B, 1, page, D, 4)
    table[0, 1], table[1, 0], table[2, 2] = -1, 10 ** 9, table.max() + 50
    cos, sin = angles(50, 64)                               # positions 50 .. 63 have a place but no angle: NaN keys
    run_append(dd, raw, table, rows(g, B, N, 1, D), rows(g, B, N, 1, D), [0, 3, 20, -7, 45, 2 ** 31 - 5], count=[33, 100, 20, 33, 33, 33],
               cos=cos, sin=sin)


def test_append_bytes_elsewhere_stay(dd):
    g = np.random.default_rng(6)
    table, raw = state(7, 2, 2, 32, 128, 3)
    before = raw[0][0].view(torch.uint8).clone(), raw[1][0].view(torch.uint8).clone()
    cache = run_append(dd, raw, table, rows(g, 2, 5, 2, 128), rows(g, 2, 5, 2, 128), [30, 64], kv_len=[30, 70])
    written = torch.zeros(raw[0][0].shape[0], 32, dtype=torch.bool)
    for b, (lo, hi) in enumerate(((30, 35), (64, 70))):
        for t in range(lo // 32 * 32, hi):
            written[table[b, t // 32], t % 32] = True
    for x, old in zip((cache.k, cache.v), before):
        same = (x.view(torch.uint8).cpu() == old).all(-1).all(1)
        assert same[~written].all()


def test_append_extremes(dd):
    """Zeros, the largest bf16 numbers, infinities, NaN, subnormal results."""
    D, page, N = 64, 16, 8
    table, raw = state(9, 1, 2, page, D, 1)
    k = torch.zeros(1, N, 2, D, dtype=torch.bfloat16)
    k[0, 1, 0, 3] = float("nan")
    k[0, 2, 0, :8] = torch.tensor([448.0, 1.0, 2.0 ** -7, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -10, -2.0 ** -11, 449.0])
    v = torch.zeros(1, N, 2, D, dtype=torch.bfloat16)
    v[0, 0, 0, :4] = torch.tensor([1e30, 1e-30, -1e20, 3e20])
    v[0, 3, 1, 0] = 2.0 ** -100
    cache = run_append(dd, raw, table, k, v, [0])
    assert float(cache.k_scale[table[0, 0], 1]) == 2.0 ** -60            # nothing but zeros
    v[0, 0, 0, 0] = float("inf")
    cache = dd.Cache(raw[0][0].cuda(), raw[1][0].cuda(), raw[0][1].cuda(), raw[1][1].cuda())
    dd.cache_append(k.cuda(), v.cuda(), cache, torch.from_numpy(table).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert float(cache.v.float()[table[0, 0], 0, 0, 0]) == 448.0 and float(cache.v_scale[table[0, 0], 0]) == 2.0 ** 60


def test_append_scales_that_are_no_powers_of_two(dd):
    """A cache quantised elsewhere: its scale is rounded up when tokens join it, its tokens move with it."""
    g = np.random.default_rng(11)
    table, raw = state(12, 2, 2, 32, 128, 2)
    raw = [(x, s * 1.37) for x, s in raw]
    run_append(dd, raw, table, rows(g, 2, 4, 2, 128), rows(g, 2, 4, 2, 128), [5, 40], kv_len=[20, 40])


@pytest.mark.parametrize("page", [16, 128])
def test_append_to_pages_under_large_scales(dd, page):
    """Scales beyond those that an append makes (a cache quantised elsewhere) stay where tokens of the page stay."""
    g = np.random.default_rng(page)
    table, raw = state(21, 2, 2, page, 64, 2)
    raw = [(x, torch.from_numpy(2.0 ** g.choice([-100, -61, 60, 61, 62, 75, 100], size=tuple(s.shape))).float()) for x, s in raw]
    raw = [(x, s * (1 + 0.5 * torch.from_numpy(g.integers(0, 2, size=tuple(s.shape))).float() * (s < 2.0 ** 99))) for x, s in raw]
    run_append(dd, raw, table, rows(g, 2, 4, 2, 64), rows(g, 2, 4, 2, 64), [5, 9], kv_len=[12, 14])


@pytest.mark.parametrize("D,dims,interleaved", [(64, 64, False), (128, 128, False), (128, 64, True), (128, 0, False)])
def test_a_row_is_the_same_whoever_computes_it(dd, D, dims, interleaved):
    """Norm and rotation in a call of one token, of many, and on the way into a cache: the same 32-bit numbers, so the same roundings."""
    g = np.random.default_rng(D + dims)
    B, N, heads, page = 2, 700, 6, 64
    k, w = rows(g, B, N, heads, D, spread=2).cuda(), weight_of(g, D).cuda()
    cos, sin = (t.cuda() for t in angles(N, dims)) if dims else (None, None)
    call = lambda x, at: dd.qk_norm_rope(x, q_weight=w, eps=EPS, cos=cos, sin=sin, interleaved=interleaved,  # noqa: E731
                                         start=torch.full((B,), at, dtype=torch.int32, device="cuda"))[0]
    many = call(k, 0)
    for i in range(0, N, 50):
        assert torch.equal(call(k[:, i:i + 1], i), many[:, i:i + 1])
    # into a cache: the e4m3 numbers next to the 32-bit results are those next to the bf16 ones, where these are not half-way between two
    wide = -(-N // page)
    table = torch.arange(B * wide, dtype=torch.int32, device="cuda").view(B, wide)
    at = torch.zeros(B, dtype=torch.int32, device="cuda")
    whole = dd.cache_append(k, k, dd.new_cache(B * wide, heads, page, D), table, at, k_weight=w, eps=EPS, cos=cos, sin=sin, interleaved=interleaved)
    single = dd.new_cache(B * wide, heads, page, D)
    for i in range(N):
        dd.cache_append(k[:, i:i + 1], k[:, i:i + 1], single, table, at + i, k_weight=w, eps=EPS, cos=cos, sin=sin, interleaved=interleaved)
    assert torch.equal(whole.k_scale, single.k_scale) and torch.equal(whole.v_scale, single.v_scale)
    order = lambda x: x.float().view(B, wide, heads, page, D).transpose(2, 3).reshape(B, wide * page, heads, D)[:, :N].double().cpu().numpy()  # noqa: E731
    scale = whole.k_scale.view(B, wide, 1, heads, 1).expand(B, wide, page, heads, 1).reshape(B, wide * page, heads, 1)[:, :N].double().cpu().numpy()
    x = many.double().cpu().numpy() / scale
    got = order(whole.k)
    lower, upper = ref.to_e4m3(x * (1 - 2.0 ** -8)), ref.to_e4m3(x * (1 + 2.0 ** -8))
    sure = lower == upper
    assert sure.mean() > 0.8 and (got[sure] == lower[sure]).all()
    middle = (x != 0) & (np.abs(x) < 448) & (ref.to_e4m3(x * (1 - 2.0 ** -20)) != ref.to_e4m3(x * (1 + 2.0 ** -20)))
    assert (got[~middle] == ref.to_e4m3(x)[~middle]).all()


def test_append_again_changes_nothing(dd):
    g = np.random.default_rng(13)
    table, raw = state(14, 3, 2, 64, 128, 3)
    k, v = rows(g, 3, 70, 2, 128), rows(g, 3, 70, 2, 128)
    cache = run_append(dd, raw, table, k, v, [0, 50, 100], kv_len=[10, 150, 100])
    again = [t.clone() for t in cache]
    dd.cache_append(k.cuda(), v.cuda(), cache, torch.from_numpy(table).cuda(), torch.tensor([0, 50, 100], dtype=torch.int32).cuda(),
                    kv_len=torch.tensor([170, 170, 170], dtype=torch.int32).cuda())
    for a, b in zip(again, cache):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_strided_projections(dd):
    g = np.random.default_rng(15)
    table, raw = state(16, 2, 4, 16, 64, 4)
    fused = rows(g, 2, 9, 3 * 4 * 64)
    k, v = fused[..., 256:512].view(2, 9, 4, 64), fused[..., 512:].view(2, 9, 4, 64)
    a = run_append(dd, raw, table, k.contiguous(), v.contiguous(), [3, 20])
    on = fused.cuda()
    cache = dd.Cache(raw[0][0].cuda(), raw[1][0].cuda(), raw[0][1].cuda(), raw[1][1].cuda())
    dd.cache_append(on[..., 256:512].view(2, 9, 4, 64), on[..., 512:].view(2, 9, 4, 64), cache, torch.from_numpy(table).cuda(),
                    torch.tensor([3, 20], dtype=torch.int32, device="cuda"))
    for x, y in zip(a, cache):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_on_another_stream_behind_what_makes_the_inputs(dd):
    """Calls on a given stream, the inputs made there just before."""
    g = np.random.default_rng(17)
    table, raw = state(18, 2, 2, 32, 128, 4)
    k, v = rows(g, 2, 40, 2, 128), rows(g, 2, 40, 2, 128)
    want = run_append(dd, raw, table, k, v, [0, 7])
    cos, sin = (t.cuda() for t in angles(64, 128))
    want_q = dd.qk_norm_rope(k.cuda(), cos=cos, sin=sin)[0]
    side = torch.cuda.Stream()
    cache = dd.Cache(raw[0][0].cuda(), raw[1][0].cuda(), raw[0][1].cuda(), raw[1][1].cuda())
    tab, start = torch.from_numpy(table).cuda(), torch.tensor([0, 7], dtype=torch.int32, device="cuda")
    dk, dv = k.cuda(), v.cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        a, b = torch.zeros_like(dk), torch.zeros_like(dv)
        for _ in range(20):
            a.add_(0)
        a.copy_(dk)
        b.copy_(dv)
    dd.cache_append(a, b, cache, tab, start, stream=side)
    got_q = dd.qk_norm_rope(a, cos=cos, sin=sin, stream=side)[0]
    torch.cuda.synchronize()
    for x, y in zip(want, cache):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert torch.equal(got_q, want_q)


def test_native_and_python_host_sides_agree(dd):
    g = np.random.default_rng(19)
    table, raw = state(20, 2, 2, 16, 64, 3)
    k, v, w = rows(g, 2, 9, 2, 64).cuda(), rows(g, 2, 9, 2, 64).cuda(), weight_of(g, 64).cuda()
    cos, sin = (t.cuda() for t in angles(64, 32))
    tab, start = torch.from_numpy(table).cuda(), torch.tensor([1, 12], dtype=torch.int32, device="cuda")
    count = torch.tensor([9, 4], dtype=torch.int32, device="cuda")
    assert dd._fast is not None
    saved, got = dd._fast, []
    try:
        for dd._fast in (saved, None):
            cache = dd.Cache(raw[0][0].cuda(), raw[1][0].cuda(), raw[0][1].cuda(), raw[1][1].cuda())
            q, kk = dd.qk_norm_rope(k, v, q_weight=w, k_weight=w, cos=cos, sin=sin, start=start, interleaved=True, layout="bhnd")
            dd.cache_append(k, v, cache, tab, start, count=count, kv_len=start, k_weight=w, cos=cos, sin=sin)
            out = dd.cached_attention(q, cache, tab, start + count, layout="bhnd", scale=0.3)
            got.append([q, kk, out, *(x.view(torch.uint8) for x in cache)])
    finally:
        dd._fast = saved
    for x, y in zip(*got):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_refusals_name_what_is_wrong(dd):
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    cos, sin = (t.cuda() for t in angles(8, 32))
    with pytest.raises(ValueError, match="both or neither"):
        dd.qk_norm_rope(q, cos=cos)
    with pytest.raises(ValueError, match="sin"):
        dd.qk_norm_rope(q, cos=cos, sin=sin[:4])
    with pytest.raises(ValueError, match="q_weight"):
        dd.qk_norm_rope(q, q_weight=torch.ones(64, device="cuda"))
    with pytest.raises(ValueError, match="out_k: given without k"):
        dd.qk_norm_rope(q, out_k=q)
    with pytest.raises(ValueError, match="k: expected"):
        dd.qk_norm_rope(q, torch.zeros(1, 5, 2, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(dd.DualDiffError):
        dd.qk_norm_rope(torch.zeros(1, 4, 2, 68, dtype=torch.bfloat16, device="cuda")[..., :64].transpose(1, 2).transpose(1, 2))
    with pytest.raises(dd.DualDiffError):
        dd.qk_norm_rope(q, eps=-1.0)
    c = dd.new_cache(4, 2, 16, 64)
    table, start = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="page_table"):
        dd.cache_append(q, q, c, table.long(), start)
    with pytest.raises(ValueError, match="v: expected"):
        dd.cache_append(q, q[:, :3], c, table, start)
    with pytest.raises(ValueError, match="cache.k_scale"):
        dd.cache_append(q, q, c._replace(k_scale=c.k_scale[:2]), table, start)
    with pytest.raises(TypeError, match="start"):
        dd.cache_append(q, q, c, table, None)
    with pytest.raises(ValueError, match="count"):
        dd.cache_append(q, q, c, table, start, count=start.float())
    with pytest.raises(dd.DualDiffError):
        dd.cache_append(q, q, dd.new_cache(4, 2, 24, 64), table, start)
