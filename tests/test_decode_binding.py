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
