"""Host side of the decoding and scoring calls: descriptor checks, sizes and refusals, all before a device is touched."""
import ctypes

import pytest

GOOD, BAD, ODD = 0x10000, 0x10008, 0x10002        # never dereferenced: 16-byte aligned, 8, 2


@pytest.fixture(scope="module")
def peqa():
    from paper_2305_14152_amd import peqa as p
    p.lib()
    return p


def cache(peqa, **changes):
    d = dict(k=GOOD, v=GOOD, table=GOOD, k_scale=None, v_scale=None, page_stride=2 * 16 * 128, head_stride=16 * 128, slot_stride=128,
             table_stride=4, n_pages=8, page_size=16, kv_heads=2, head_dim=128, n_seqs=3, n_blocks=4, dtype=0, reserved=0)
    d.update(changes)
    return peqa.KVCache(**d)


def test_descriptors(peqa):
    assert peqa.check_cache(cache(peqa)) == peqa.PEQA_OK
    assert peqa.lib().peqa_check_cache(None) == peqa.PEQA_ERR_NULL
    fp8 = dict(dtype=1, k_scale=GOOD, v_scale=GOOD)
    assert peqa.check_cache(cache(peqa, **fp8)) == peqa.PEQA_OK
    for bad, status in [(dict(k=None), 1), (dict(v=None), 1), (dict(table=None), 1), (dict(dtype=2), 8), (dict(dtype=-1), 8),
                        (dict(reserved=1), 8), (dict(k_scale=GOOD), 8), (dict(page_size=24), 2), (dict(page_size=4), 2),
                        (dict(page_size=2048), 2), (dict(page_size=0), 2), (dict(head_dim=80), 2), (dict(head_dim=512), 2),
                        (dict(n_pages=0), 2), (dict(kv_heads=0), 2), (dict(n_seqs=0), 2), (dict(n_blocks=0), 2),
                        (dict(n_blocks=1 << 28, table_stride=1 << 28), 2), (dict(table_stride=3), 2), (dict(page_stride=-8), 2),
                        (dict(head_stride=-8), 2), (dict(slot_stride=120), 2), (dict(k=BAD), 5), (dict(v=BAD), 5),
                        (dict(table=ODD), 5), (dict(page_stride=4100), 5), (dict(slot_stride=132), 5),
                        (dict(fp8, head_stride=16 * 128 + 8), 5), (dict(fp8, v_scale=ODD), 5)]:
        assert peqa.check_cache(cache(peqa, **bad)) == status, bad


def test_append_refusals(peqa):
    L = peqa.lib()
    C = cache(peqa)

    def call(**changes):
        d = dict(C=C, T=3, pos=GOOD, seq=None, cos=GOOD, sin=GOOD, n_pos=64, rot=128, il=0, heads=4, q=GOOD, qs=512, k=GOOD, ks=256,
                 v=GOOD, vs=256, o=GOOD, os=512, stream=None)
        d.update(changes)
        return L.peqa_rope_append(*d.values())

    for bad, status in [(dict(C=None), 1), (dict(C=cache(peqa, head_dim=100)), 2), (dict(pos=None), 1), (dict(k=None), 1), (dict(v=None), 1),
                        (dict(q=None), 1), (dict(o=None), 1), (dict(cos=None), 1), (dict(sin=None), 1), (dict(T=0), 2), (dict(T=-1), 2),
                        (dict(T=4), 2), (dict(heads=0), 2), (dict(rot=144), 8), (dict(rot=24), 8), (dict(rot=-16), 8), (dict(n_pos=0), 8),
                        (dict(qs=504), 2), (dict(ks=248), 2), (dict(vs=248), 2), (dict(os=504), 2), (dict(q=BAD), 5), (dict(k=BAD), 5),
                        (dict(v=BAD), 5), (dict(o=BAD), 5), (dict(qs=516), 5), (dict(ks=260), 5), (dict(vs=260), 5), (dict(os=516), 5),
                        (dict(cos=BAD), 5), (dict(sin=BAD), 5), (dict(pos=ODD), 5), (dict(seq=ODD), 5),
                        (dict(seq=GOOD, T=2 ** 31 - 1), 2)]:
        assert call(**bad) == status, bad


def test_attention_refusals_and_sizes(peqa):
    L = peqa.lib()
    C = cache(peqa)

    def call(**changes):
        d = dict(C=C, rows=3, heads=4, q=GOOD, qs=512, lens=GOOD, seq=None, most=64, window=0, scale=0.1, o=GOOD, os=512, lse=GOOD,
                 ws=GOOD, room=1 << 20, stream=None)
        d.update(changes)
        return L.peqa_paged_attention(*d.values())

    for bad, status in [(dict(C=None), 1), (dict(C=cache(peqa, page_size=12)), 2), (dict(q=None), 1), (dict(lens=None), 1), (dict(o=None), 1),
                        (dict(rows=0), 2), (dict(heads=3), 2), (dict(heads=0), 2), (dict(most=65), 2), (dict(most=-1), 2), (dict(window=-1), 8),
                        (dict(rows=4), 2), (dict(qs=504), 2), (dict(os=504), 2), (dict(qs=516), 5), (dict(os=516), 5), (dict(q=BAD), 5),
                        (dict(o=BAD), 5), (dict(lens=ODD), 5), (dict(seq=ODD), 5), (dict(lse=ODD), 5)]:
        assert call(**bad) == status, bad
    long = cache(peqa, n_blocks=1 << 16, table_stride=1 << 16)
    need = peqa.paged_attention_workspace_bytes(long, 4, 1, 1 << 20)
    assert need > 256
    assert call(C=long, rows=1, most=1 << 20, ws=None) == peqa.PEQA_ERR_WORKSPACE
    assert call(C=long, rows=1, most=1 << 20, room=need - 1) == peqa.PEQA_ERR_WORKSPACE
    assert call(C=long, rows=1, most=1 << 20, room=need, ws=BAD) == peqa.PEQA_ERR_ALIGN
    # a window bounds what there is to split
    assert peqa.paged_attention_workspace_bytes(long, 4, 1, 1 << 20, 64) <= peqa.paged_attention_workspace_bytes(long, 4, 1, 128)
    assert peqa.paged_attention_workspace_bytes(C, 3, 1, 64) == 0
    assert peqa.paged_attention_workspace_bytes(C, 4, 1, 65) == 0


def test_logprob_refusals_and_sizes(peqa):
    L = peqa.lib()

    def call(**changes):
        d = dict(x=GOOD, dtype=0, T=3, V=1000, stride=1000, t=GOOD, top=5, logp=GOOD, H=GOOD, lse=GOOD, tl=GOOD, ti=GOOD, ws=GOOD, room=1 << 20,
                 stream=None)
        d.update(changes)
        return L.peqa_token_logprobs(*d.values())

    for bad, status in [(dict(x=None), 1), (dict(t=None), 1), (dict(tl=None), 1), (dict(ti=None), 1), (dict(logp=None, H=None, lse=None, top=0), 1),
                        (dict(dtype=2), 8), (dict(T=0), 2), (dict(V=0), 2), (dict(V=(1 << 30) + 1, stride=1 << 31), 2), (dict(stride=999), 2),
                        (dict(top=33), 8), (dict(top=-1), 8), (dict(top=6, V=5), 8), (dict(x=0x10001), 5), (dict(x=ODD, dtype=1), 5),
                        (dict(t=ODD), 5), (dict(logp=ODD), 5), (dict(ti=ODD), 5)]:
        assert call(**bad) == status, bad
    need = peqa.token_logprobs_workspace_bytes(1, 200000, 32)
    assert need > 256
    assert call(T=1, V=200000, stride=200000, top=32, room=need - 1) == peqa.PEQA_ERR_WORKSPACE
    assert call(T=1, V=200000, stride=200000, top=32, ws=None) == peqa.PEQA_ERR_WORKSPACE
    assert call(T=1, V=200000, stride=200000, top=32, room=need, ws=BAD) == peqa.PEQA_ERR_ALIGN
    assert peqa.token_logprobs_workspace_bytes(0, 100, 0) == 0 and peqa.token_logprobs_workspace_bytes(1, 100, 33) == 0
    assert peqa.token_logprobs_workspace_bytes(4096, 32000, 20) > 0

    def back(**changes):
        d = dict(x=GOOD, dtype=0, T=3, V=1000, stride=1000, t=GOOD, lse=GOOD, H=GOOD, g=GOOD, h=GOOD, d=2 * GOOD, ds=1000, stream=None)
        d.update(changes)
        return L.peqa_token_logprobs_bwd(*d.values())

    for bad, status in [(dict(x=None), 1), (dict(lse=None), 1), (dict(d=None), 1), (dict(g=None, h=None), 1), (dict(t=None), 1), (dict(H=None), 1),
                        (dict(dtype=-1), 8), (dict(T=-2), 2), (dict(V=0), 2), (dict(stride=10), 2), (dict(ds=10), 2),
                        (dict(d=GOOD, ds=1008), 2), (dict(d=0x20001), 5), (dict(g=ODD), 5)]:
        assert back(**bad) == status, bad


def test_binding_checks(peqa):
    import torch
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    table = torch.zeros((3, 4), dtype=torch.int32)
    c = peqa.kv_cache(k, k.clone(), table)
    assert peqa.check_cache(c) == peqa.PEQA_OK and c.page_stride == 4096 and c.dtype == peqa.PEQA_CACHE_BF16
    assert peqa.kv_cache(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn), table).dtype == peqa.PEQA_CACHE_FP8
    with pytest.raises(AssertionError):
        peqa.kv_cache(k, k.transpose(2, 3), table)
    with pytest.raises(AssertionError):
        peqa.kv_cache(k, k.clone(), table.long())
    q = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(peqa.PeqaError) as e:                      # more rows than sequences
        peqa.paged_attention(c, q, torch.zeros(4, dtype=torch.int32), 64, 1.0, q.clone(), None, 0, stream=0)
    assert e.value.status == peqa.PEQA_ERR_SHAPE
    with pytest.raises(AssertionError):
        peqa.paged_attention(c, q.transpose(1, 2), torch.zeros(4, dtype=torch.int32), 64, 1.0, q.clone(), None, 0, stream=0)
    assert ctypes.sizeof(peqa.KVCache) == 104


def test_sizes_past_what_the_kernels_index(peqa):
    """Positions past 2^30, units of a row past 2^30 and launches of more than 2^32 threads are refused."""
    L = peqa.lib()
    assert peqa.check_cache(cache(peqa, n_blocks=1 << 26, table_stride=1 << 26)) == peqa.PEQA_OK
    assert peqa.check_cache(cache(peqa, n_blocks=(1 << 26) + 1, table_stride=1 << 27)) == peqa.PEQA_ERR_SHAPE
    wide = cache(peqa, n_blocks=1 << 26, table_stride=1 << 26, kv_heads=128, page_stride=128 * 16 * 128)
    assert peqa.paged_attention_workspace_bytes(wide, 128, 1, 1 << 30) == 0 and peqa.paged_attention_workspace_bytes(wide, 128, 1, 1 << 28) > 0
    many = cache(peqa, kv_heads=64, n_seqs=1 << 30, page_stride=64 * 16 * 128)
    assert peqa.paged_attention_workspace_bytes(many, 64, 1 << 20, 16) == 0
    assert L.peqa_token_logprobs(GOOD, 0, 1 << 24, 100, 100, GOOD, 0, GOOD, None, None, None, None, None, 0, None) == peqa.PEQA_ERR_SHAPE
    assert L.peqa_token_logprobs_bwd(GOOD, 0, 1 << 20, 1 << 20, 1 << 20, GOOD, GOOD, None, GOOD, None, 2 * GOOD, 1 << 20, None) == peqa.PEQA_ERR_SHAPE
