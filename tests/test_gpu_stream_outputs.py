"""Calls on a stream of their own: the outputs that a call makes are memory of that stream, not memory that the current stream still reads."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dd():
    from paper_2604_05250_b200 import binding, build
    build.build()
    return binding


def calls(dd):
    """name -> (call on a stream, sizes in bytes of the outputs that it makes)"""
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    B, N, H, D, V, K = 2, 512, 4, 128, 1000, 64
    q, k, v = bf(B, H, N, D), bf(B, H, N, D), bf(B, H, N, D)
    cache = dd.new_cache(B * N // 64, H, 64, D)
    table = torch.arange(B * N // 64, dtype=torch.int32, device="cuda").view(B, -1)
    lens = torch.full((B,), N, dtype=torch.int32, device="cuda")
    P = 2048
    logits, drafter = bf(1, P, V), bf(1, P, V)
    tokens, flags = torch.zeros(1, P, dtype=torch.int32, device="cuda"), torch.ones(1, P, dtype=torch.uint8, device="cuda")
    hidden, weight = bf(1, P, K), bf(V, K)
    rows, ints, marks = B * H * N * D * 2, P * 4, P
    return {
        "bidir_attention": (lambda s: dd.bidir_attention(q, k, v, stream=s), [rows]),
        "block_attention": (lambda s: dd.block_attention(q, k, v, kv_len=lens, stream=s), [rows]),
        "verify": (lambda s: dd.verify(drafter, logits, tokens, flags, 1, 0.1, 0, 1, stream=s), [ints, marks, ints]),
        "unmask": (lambda s: dd.unmask(logits, tokens, flags, 0.5, 1, stream=s), [ints, marks, ints]),
        "lm_head_verify": (lambda s: dd.lm_head_verify(None, None, hidden, weight, tokens, flags, 2, 0.5, 0, 1, stream=s), [ints, marks, ints]),
        "qk_norm_rope": (lambda s: dd.qk_norm_rope(q, k, layout="bhnd", stream=s), [rows, rows]),
        "cached_attention": (lambda s: dd.cached_attention(q, cache, table, lens, layout="bhnd", stream=s), [rows]),
    }


@pytest.mark.parametrize("name", ["bidir_attention", "block_attention", "verify", "unmask", "lm_head_verify", "qk_norm_rope", "cached_attention"])
def test_memory_that_the_current_stream_still_reads(dd, name):
    """Blocks as large as the outputs are freed while a copy out of them is still queued on the current stream, which is theirs: a call
    on another stream must not write there."""
    call, sizes = calls(dd)[name]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = call(side)                                   # (scratch of the library exists from here on)
    torch.cuda.synchronize()
    want = [x.clone() for x in (want if isinstance(want, tuple) else (want,)) if x is not None]
    torch.cuda.synchronize()
    blocks = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in sizes]
    copies = [torch.empty_like(b) for b in blocks]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                       # some 50 ms
    for b, c in zip(blocks, copies):
        c.copy_(b)
    del b, blocks                                        # free for later work on the current stream
    got = call(side)
    torch.cuda.synchronize()
    assert all((c == 0x5A).all() for c in copies)
    got = [x for x in (got if isinstance(got, tuple) else (got,)) if x is not None]
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_an_output_on_another_stream_outlives_its_owner(dd):
    """The other way round: an output that is dropped while its stream still writes it is not given to the current stream."""
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(1, 4, 512, 128, generator=g, device="cuda").bfloat16()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    dd.qk_norm_rope(q, stream=side)
    mine = [torch.full((1, 512, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all((x == 3).all() for x in mine)


@pytest.mark.parametrize("name", ["bidir_attention", "block_attention", "verify", "unmask", "lm_head_verify", "qk_norm_rope", "cached_attention"])
def test_a_stream_that_is_not_torchs(dd, name):
    """Anything with a cuda_stream is a stream to these calls."""
    class Other:
        def __init__(self, pointer):
            self.cuda_stream = pointer
    call, _ = calls(dd)[name]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for pointer in (side.cuda_stream, 0):
        got, want = call(Other(pointer)), call(None)
        torch.cuda.synchronize()
        for x, y in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
            assert torch.equal(x, y)
