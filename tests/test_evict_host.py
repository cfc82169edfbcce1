"""Host side of the accumulating attention and of eviction: sizes and refusals, all before a device is touched."""
import pytest

from test_decode_host import BAD, GOOD, ODD, cache


@pytest.fixture(scope="module")
def peqa():
    from paper_2305_14152_amd import peqa as p
    p.lib()
    return p


def test_attention_refusals_and_sizes(peqa):
    L, C = peqa.lib(), cache(peqa)

    def call(**changes):
        d = dict(C=C, rows=3, heads=4, q=GOOD, qs=512, lens=GOOD, seq=None, most=64, window=0, scale=0.1, o=GOOD, os=512, lse=GOOD, w=GOOD, wo=GOOD,
                 ss=128, hs=64, ws=GOOD, room=1 << 20, stream=None)
        d.update(changes)
        return L.peqa_paged_attention_weights(*d.values())

    for bad, status in [(dict(C=None), 1), (dict(q=None), 1), (dict(lens=None), 1), (dict(o=None), 1), (dict(wo=None), 1), (dict(rows=0), 2), (dict(heads=3), 2),
                        (dict(most=65), 2), (dict(rows=4), 2), (dict(qs=504), 2), (dict(window=-1), 8), (dict(hs=60), 2), (dict(ss=60), 2),
                        (dict(hs=66), 5), (dict(ss=130), 5), (dict(w=BAD), 5), (dict(wo=BAD), 5), (dict(q=BAD), 5), (dict(lse=ODD), 5), (dict(ws=None), 6),
                        (dict(ws=BAD), 5)]:
        assert call(**bad) == status, bad
    need = peqa.paged_attention_weights_workspace_bytes(C, 4, 3, 64)
    assert need >= 4 * 3 * 4 * 65 and call(room=need - 1) == peqa.PEQA_ERR_WORKSPACE
    assert need >= peqa.paged_attention_workspace_bytes(C, 4, 3, 64) - 256
    assert peqa.paged_attention_weights_workspace_bytes(C, 3, 3, 64) == 0 and peqa.paged_attention_weights_workspace_bytes(C, 4, 3, 65) == 0
    long = cache(peqa, n_blocks=1 << 16, table_stride=1 << 16, n_seqs=1 << 20, kv_heads=1, head_stride=0)
    assert call(C=long, rows=1 << 17, seq=GOOD, heads=1, qs=128, os=128, most=1 << 20, hs=1 << 20, ss=1 << 20, room=1 << 50) == peqa.PEQA_ERR_SHAPE


def test_eviction_refusals_and_sizes(peqa):
    L, C = peqa.lib(), cache(peqa)

    def call(**changes):
        d = dict(C=C, to=None, n=3, seq=None, lens=GOOD, most=64, w=GOOD, wo=GOOD, ss=128, hs=64, keep=30, sinks=4, recent=10, kept=GOOD, new=2 * GOOD, ws=GOOD,
                 room=1 << 20, stream=None)
        d.update(changes)
        return L.peqa_cache_evict(*d.values())

    other = dict(k=3 * GOOD, v=3 * GOOD, table=3 * GOOD)
    for bad, status in [(dict(C=None), 1), (dict(C=cache(peqa, page_size=12)), 2), (dict(lens=None), 1), (dict(w=None), 1), (dict(wo=None), 1), (dict(n=0), 2),
                        (dict(n=4), 2), (dict(most=65), 2), (dict(most=-1), 2), (dict(keep=0), 8), (dict(keep=-5), 8), (dict(keep=(1 << 30) + 1), 8),
                        (dict(sinks=-1), 8), (dict(recent=-1), 8), (dict(sinks=21), 8), (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), 8),
                        (dict(new=GOOD), 8), (dict(hs=63), 2), (dict(ss=63), 2), (dict(lens=ODD), 5), (dict(seq=ODD), 5), (dict(w=ODD), 5), (dict(wo=ODD), 5),
                        (dict(kept=ODD), 5), (dict(new=ODD), 5), (dict(ws=None), 6), (dict(ws=BAD), 5), (dict(n=1 << 20, seq=GOOD), 2),
                        (dict(to=cache(peqa, **other, kv_heads=1)), 2), (dict(to=cache(peqa, **other, head_dim=64)), 2), (dict(to=cache(peqa, **other, n_seqs=4)), 2),
                        (dict(to=cache(peqa, **other, dtype=1)), 8), (dict(to=cache(peqa, **other, page_size=24)), 2),
                        (dict(to=cache(peqa, **other, n_blocks=1)), 2), (dict(to=cache(peqa, page_size=8)), 8), (dict(to=cache(peqa, head_stride=8 * 128)), 8),
                        (dict(to=cache(peqa, table_stride=5)), 8)]:
        assert call(**bad) == status, bad
    need = peqa.cache_evict_workspace_bytes(C, 3, 64, 30)
    assert need >= 4 * (3 * 2 * 30 + 3) and call(room=need - 1) == peqa.PEQA_ERR_WORKSPACE
    assert peqa.cache_evict_workspace_bytes(C, 0, 64, 30) == 0 and peqa.cache_evict_workspace_bytes(C, 3, 65, 30) == 0
    assert peqa.cache_evict_workspace_bytes(C, 3, 64, 0) == 0
    # lengths that the call would read and write; more workgroups than a launch has
    for behind in (4, -8):
        assert call(new=GOOD + behind) == peqa.PEQA_ERR_PARAM
    long = cache(peqa, n_blocks=1 << 16, table_stride=1 << 16, n_seqs=1 << 20, kv_heads=1, head_stride=0)
    many = dict(C=long, n=1 << 20, seq=GOOD, most=1 << 20, hs=1 << 20, ss=1 << 20, keep=1 << 20, kept=None, new=None, room=1 << 50)
    assert call(**many) == peqa.PEQA_ERR_SHAPE and peqa.cache_evict_workspace_bytes(long, 1 << 20, 1 << 20, 1 << 20) == 0


def test_binding(peqa):
    import torch
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    table, index, w = torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, 64)
    c = peqa.kv_cache(k, k.clone(), table)
    q = torch.zeros((3, 4, 128), dtype=torch.bfloat16)
    attend = dict(cache=c, q=q, lens=index, max_len=64, scale=1.0, out=q.clone(), weights=w, weights_out=w.clone(), workspace=None, workspace_bytes_=0, stream=0)
    evict = dict(cache=c, lens=index, max_len=64, weights=w, weights_out=w.clone(), keep=8, sinks=1, recent=2,
                 kept=torch.zeros((3, 2, 8), dtype=torch.int32), new_lens=index.clone(), workspace=None, workspace_bytes_=0, stream=0)
    for name, good in (("paged_attention_weights", attend), ("cache_evict", evict)):
        call = getattr(peqa, name)
        with pytest.raises(peqa.PeqaError) as e:
            call(**good)
        assert e.value.status == peqa.PEQA_ERR_WORKSPACE
        for bad in (dict(weights=w.double()), dict(weights=w[:2]), dict(weights_out=w.bfloat16()), dict(weights=torch.zeros(3, 2, 128)[:, :, ::2]),
                    dict(weights_out=torch.zeros(3, 2, 128)[..., :64]), dict(weights=w[..., :63].clone(), weights_out=w[..., :63].clone()),
                    dict(weights=w[:1].expand(3, 2, 64), weights_out=w[:1].expand(3, 2, 64)), dict(lens=index.long()), dict(seq=index.float()), dict(seq=index[:2]),
                    dict(workspace=torch.zeros(8, dtype=torch.uint8), workspace_bytes_=16)):
            with pytest.raises(AssertionError):
                call(**{**good, **bad})
    for bad in (dict(kept=torch.zeros((3, 2, 9), dtype=torch.int32)), dict(kept=torch.zeros((3, 2, 8))), dict(new_lens=index), dict(new_lens=index[:2].clone()),
                dict(weights=None), dict(to=peqa.kv_cache(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn), table, torch.ones(2), None))):
        with pytest.raises(AssertionError):
            peqa.cache_evict(**{**evict, **bad})
