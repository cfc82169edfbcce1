"""What the Python side of the decoding and scoring calls refuses before the library is called, and what it lets through.  No tensor's
memory is read: everything is decided from shapes, strides and types."""
import pytest


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


def pools(torch, kind=None):
    k = torch.zeros((4, 2, 16, 128), dtype=kind or torch.bfloat16)
    return k, torch.zeros_like(k)


def test_tables_whose_rows_overlap(env):
    """The descriptor's rows are at least a row's entries apart: what is closer would be read past its end."""
    torch, peqa = env
    k, v = pools(torch)
    row = torch.zeros((1, 4), dtype=torch.int32)
    for table in (row.expand(3, -1), torch.zeros(8, dtype=torch.int32).as_strided((3, 4), (2, 1)),
                  torch.zeros(8, dtype=torch.int32).as_strided((2, 4), (3, 1))):
        with pytest.raises(AssertionError, match="table"):
            peqa.kv_cache(k, v, table)
    # a single row may have any stride; rows further apart are as they are
    assert peqa.kv_cache(k, v, row.expand(1, -1)).table_stride == 4
    assert peqa.kv_cache(k, v, torch.zeros(4, dtype=torch.int32).as_strided((1, 4), (0, 1))).table_stride == 4
    assert peqa.kv_cache(k, v, torch.zeros((3, 9), dtype=torch.int32)[:, :4]).table_stride == 9
    assert peqa.kv_cache(k, v, torch.zeros((3, 4), dtype=torch.int32)).table_stride == 4


def test_types_of_pools_and_table(env):
    """8-bit pools are e4m3fn (or its bytes), 16-bit ones bf16 (or its 16-bit patterns), tables int32: nothing else of the same width."""
    torch, peqa = env
    table = torch.zeros((3, 4), dtype=torch.int32)
    for kind in (torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.int8, torch.bool, torch.float16, torch.float32):
        with pytest.raises(AssertionError, match="pools"):
            peqa.kv_cache(*pools(torch, kind), table)
    for kind in (torch.float32, torch.uint32, torch.int64, torch.int16):
        with pytest.raises(AssertionError, match="table"):
            peqa.kv_cache(*pools(torch), torch.zeros((3, 4), dtype=kind))
    for kind, want in ((torch.bfloat16, 0), (torch.int16, 0), (torch.uint16, 0), (torch.float8_e4m3fn, 1), (torch.uint8, 1)):
        c = peqa.kv_cache(*pools(torch, kind), table)
        assert c.dtype == want and peqa.check_cache(c) == peqa.PEQA_OK


def test_scales(env):
    """A scale per key head, fp32, contiguous."""
    torch, peqa = env
    k, v = pools(torch, torch.float8_e4m3fn)
    table = torch.zeros((3, 4), dtype=torch.int32)
    good = torch.ones(2)
    for bad in (torch.ones(1), torch.ones(()), torch.ones(2, dtype=torch.float64), torch.ones(2, dtype=torch.bfloat16), torch.ones(4)[::2],
                torch.ones(1).expand(2), torch.ones(3)):
        for args in ((bad, good), (good, bad)):
            with pytest.raises(AssertionError):
                peqa.kv_cache(k, v, table, *args)
    assert peqa.check_cache(peqa.kv_cache(k, v, table, good, good.clone())) == peqa.PEQA_OK
    assert peqa.check_cache(peqa.kv_cache(k, v, table, None, good)) == peqa.PEQA_OK
    assert peqa.check_cache(peqa.kv_cache(k, v, table, good.view(2, 1), None)) == peqa.PEQA_OK


def test_scales_may_be_addresses(env):
    """As elsewhere in the binding, an integer is taken for a device address."""
    torch, peqa = env
    k, v = pools(torch, torch.float8_e4m3fn)
    c = peqa.kv_cache(k, v, torch.zeros((3, 4), dtype=torch.int32), 0x10000, 0x20000)
    assert (c.k_scale, c.v_scale) == (0x10000, 0x20000) and peqa.check_cache(c) == peqa.PEQA_OK


def bound(torch, peqa):
    """A cache, its inputs for three tokens, and logits with all that the scoring calls take."""
    k, v = pools(torch)
    cache = peqa.kv_cache(k, v, torch.zeros((3, 4), dtype=torch.int32))
    bf16 = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)  # noqa: E731
    ints = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    append = dict(q=bf16(3, 4, 128), k=bf16(3, 2, 128), v=bf16(3, 2, 128), pos=ints(3), cos=torch.zeros(64, 64), sin=torch.zeros(64, 64),
                  q_out=bf16(3, 4, 128), seq=ints(3))
    attend = dict(q=bf16(3, 4, 128), lens=ints(3), max_len=64, scale=1.0, out=bf16(3, 4, 128), workspace=None, workspace_bytes_=0,
                  lse=torch.zeros(3, 4), seq=ints(3))
    score = dict(logits=bf16(3, 100), targets=ints(3), logp=torch.zeros(3), entropy=torch.zeros(3), lse=torch.zeros(3), top_logp=torch.zeros(3, 5),
                 top_ids=torch.zeros((3, 5), dtype=torch.int32), workspace=None, workspace_bytes_=0)
    back = dict(logits=bf16(3, 100), targets=ints(3), lse=torch.zeros(3), entropy=torch.zeros(3), d_logp=torch.zeros(3), d_entropy=torch.zeros(3),
                d_logits=bf16(3, 100))
    return cache, append, attend, score, back


class Called(Exception):
    pass


@pytest.fixture()
def calls(env, monkeypatch):
    """The four calls with good arguments, and a library that says that it was reached instead of launching anything."""
    torch, peqa = env
    cache, append, attend, score, back = bound(torch, peqa)

    class Library:
        def __getattr__(self, name):
            def reached(*args):
                raise Called(name)
            return reached
    monkeypatch.setattr(peqa, "_lib", Library())

    def call(name, **changes):
        first, good = {"rope_append": ((cache,), append), "paged_attention": ((cache,), attend), "token_logprobs": ((), score),
                       "token_logprobs_bwd": ((), back)}[name]
        return getattr(peqa, name)(*first, stream=0, **{**good, **changes})

    for name in ("rope_append", "paged_attention", "token_logprobs", "token_logprobs_bwd"):
        with pytest.raises(Called):
            call(name)
    return call


INDEXES = [("rope_append", "pos"), ("rope_append", "seq"), ("paged_attention", "lens"), ("paged_attention", "seq"), ("token_logprobs", "targets"),
           ("token_logprobs_bwd", "targets")]


@pytest.mark.parametrize("name,argument", INDEXES)
def test_positions_lengths_sequences_and_words_are_int32(env, calls, name, argument):
    torch, _ = env
    for bad in (torch.zeros(3, dtype=torch.int64), torch.zeros(3), torch.zeros(3, dtype=torch.int16), torch.zeros(3, dtype=torch.uint32),
                torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(AssertionError):
            calls(name, **{argument: bad})
    with pytest.raises(Called):
        calls(name, **{argument: torch.zeros((3, 1), dtype=torch.int32)})


@pytest.mark.parametrize("name,arguments", [("rope_append", ("q",)), ("rope_append", ("k",)), ("rope_append", ("v",)), ("rope_append", ("q_out",)),
                                            ("paged_attention", ("q",)), ("paged_attention", ("out",)), ("token_logprobs", ("logits",)),
                                            ("token_logprobs_bwd", ("logits", "d_logits")), ("token_logprobs_bwd", ("d_logits",))])
def test_queries_keys_values_and_logits_are_bf16(env, calls, name, arguments):
    """bf16 or its 16-bit pattern, logits also fp32: nothing else of the same width."""
    torch, peqa = env
    shape = {"k": (3, 2, 128), "v": (3, 2, 128), "logits": (3, 100), "d_logits": (3, 100)}.get(arguments[0], (3, 4, 128))
    for kind in (torch.float16, torch.int32, torch.uint8, torch.float64):
        with pytest.raises(AssertionError, match="bf16"):
            calls(name, **{a: torch.zeros(shape, dtype=kind) for a in arguments})
    for kind in (torch.bfloat16, torch.int16, torch.uint16):
        with pytest.raises(Called):
            calls(name, **{a: torch.zeros(shape, dtype=kind) for a in arguments})
    good = {a: torch.zeros(shape, dtype=torch.float32) for a in arguments}
    with pytest.raises(Called if "logits" in arguments else AssertionError):
        calls(name, **good)


@pytest.mark.parametrize("argument", ["cos", "sin"])
def test_rotation_tables_are_fp32(env, calls, argument):
    """bf16 tables, as models often keep them, would be read as half as many fp32 numbers and past their end."""
    torch, peqa = env
    for kind in (torch.bfloat16, torch.float16, torch.float64, torch.int32):
        with pytest.raises(AssertionError, match="float32"):
            calls("rope_append", **{argument: torch.zeros((64, 64), dtype=kind)})
    for bad in (torch.zeros((64, 128))[:, ::2], torch.zeros((64, 65))[:, :64], torch.zeros((64, 64)).T, torch.zeros((1, 64)).expand(64, -1)):
        with pytest.raises(AssertionError):
            calls("rope_append", **{argument: bad})
    with pytest.raises(Called):
        calls("rope_append", cos=None, sin=None)
    with pytest.raises(Called):
        calls("rope_append", cos=torch.zeros((64, 128))[:32, :64].contiguous(), sin=torch.zeros((32, 64)))


FLOATS = [("paged_attention", "lse"), ("token_logprobs", "logp"), ("token_logprobs", "entropy"), ("token_logprobs", "lse"), ("token_logprobs", "top_logp"),
          ("token_logprobs_bwd", "lse"), ("token_logprobs_bwd", "entropy"), ("token_logprobs_bwd", "d_logp"), ("token_logprobs_bwd", "d_entropy")]


@pytest.mark.parametrize("name,argument", FLOATS)
def test_numbers_of_rows_are_fp32_and_as_many(env, calls, name, argument):
    torch, _ = env
    shape = {"paged_attention": (3, 4)}.get(name, (3, 5) if argument == "top_logp" else (3,))
    for kind in (torch.bfloat16, torch.float16, torch.float64, torch.int32):
        with pytest.raises(AssertionError, match="float32"):
            calls(name, **{argument: torch.zeros(shape, dtype=kind)})
    for bad in (torch.zeros((2,) + shape[1:]), torch.zeros(()), torch.zeros((1,) + shape[1:]).expand(shape), torch.zeros((6,) + shape[1:])[::2]):
        with pytest.raises(AssertionError):
            calls(name, **{argument: bad})
    if len(shape) == 1:                            # buffers made for more rows, and device addresses
        for good in (torch.zeros(8), 0x10000):
            with pytest.raises(Called):
                calls(name, **{argument: good})


def test_alternatives_are_int32(env, calls):
    torch, _ = env
    for bad in (torch.zeros((3, 5), dtype=torch.int64), torch.zeros((3, 5)), torch.zeros((3, 10), dtype=torch.int32)[:, ::2],
                torch.zeros((2, 5), dtype=torch.int32), torch.zeros((3, 4), dtype=torch.int32)):
        with pytest.raises(AssertionError):
            calls("token_logprobs", top_ids=bad)


@pytest.mark.parametrize("name", ["paged_attention", "token_logprobs"])
def test_workspaces_are_as_large_as_they_are_said_to_be(env, calls, name):
    torch, _ = env
    for room, said in ((torch.zeros(255, dtype=torch.uint8), 256), (torch.zeros(63), 256), (torch.zeros(512, dtype=torch.uint8)[::2], 256)):
        with pytest.raises(AssertionError):
            calls(name, workspace=room, workspace_bytes_=said)
    for room, said in ((torch.zeros(256, dtype=torch.uint8), 256), (torch.zeros(64), 256), (torch.zeros(1000, dtype=torch.uint8), 256), (0x10000, 256)):
        with pytest.raises(Called):
            calls(name, workspace=room, workspace_bytes_=said)
