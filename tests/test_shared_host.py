"""Host side of the attention behind shared positions: sizes and refusals, all before a device is touched."""
import pytest

from test_decode_host import BAD, GOOD, ODD, cache


@pytest.fixture(scope="module")
def peqa():
    from paper_2305_14152_amd import peqa as p
    p.lib()
    return p


def test_refusals_and_sizes(peqa):
    L, C = peqa.lib(), cache(peqa)

    def call(**changes):
        d = dict(C=C, rows=3, heads=4, q=GOOD, qs=512, lens=GOOD, seq=None, most=64, prefix=2, shared=30, scale=0.1, o=GOOD, os=512, lse=GOOD, ws=GOOD,
                 room=1 << 20, stream=None)
        d.update(changes)
        return L.peqa_shared_attention(*d.values())

    for bad, status in [(dict(C=None), 1), (dict(C=cache(peqa, page_size=12)), 2), (dict(q=None), 1), (dict(lens=None), 1), (dict(o=None), 1), (dict(rows=0), 2),
                        (dict(heads=3), 2), (dict(heads=0), 2), (dict(most=65), 2), (dict(most=-1), 2), (dict(shared=65), 2), (dict(shared=-1), 2),
                        (dict(prefix=-1), 2), (dict(prefix=3), 2), (dict(rows=4), 2), (dict(qs=504), 2), (dict(os=504), 2), (dict(qs=516), 5), (dict(os=516), 5),
                        (dict(q=BAD), 5), (dict(o=BAD), 5), (dict(lens=ODD), 5), (dict(seq=ODD), 5), (dict(lse=ODD), 5), (dict(ws=None), 6),
                        (dict(ws=BAD), 5), (dict(rows=1 << 22, seq=GOOD), 2)]:
        assert call(**bad) == status, bad
    need = peqa.shared_attention_workspace_bytes(C, 4, 3, 64, 30)
    assert need > 0 and call(room=need - 1) == peqa.PEQA_ERR_WORKSPACE
    for rows, heads, most, shared in ((0, 4, 64, 30), (3, 3, 64, 30), (3, 4, 65, 30), (3, 4, 64, 65), (3, 4, 64, -1)):
        assert peqa.shared_attention_workspace_bytes(C, heads, rows, most, shared) == 0
    # the parts of many rows take little beside what they read
    long = cache(peqa, n_blocks=1 << 13, table_stride=1 << 13, kv_heads=8, n_seqs=300)
    for rows, shared in ((1, 1 << 17), (64, 8192), (256, 1 << 17)):
        assert 0 < peqa.shared_attention_workspace_bytes(long, 64, rows, 1 << 17, shared) <= 128 << 20


def test_binding(peqa):
    import torch
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    c = peqa.kv_cache(k, k.clone(), torch.zeros((3, 4), dtype=torch.int32))
    q, index = torch.zeros((3, 4, 128), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    good = dict(cache=c, q=q, lens=index, max_len=64, prefix=2, shared=30, scale=1.0, out=q.clone(), workspace=None, workspace_bytes_=0, lse=torch.zeros(3, 4),
                seq=index, stream=0)
    with pytest.raises(peqa.PeqaError) as e:
        peqa.shared_attention(**good)
    assert e.value.status == peqa.PEQA_ERR_WORKSPACE
    for bad in (dict(q=q.half()), dict(q=q.transpose(0, 1)), dict(out=torch.zeros((3, 4, 64), dtype=torch.bfloat16)), dict(lens=index.long()), dict(lens=index[:2]),
                dict(seq=index.float()), dict(lse=torch.zeros(3, 5)), dict(lse=torch.zeros(3, 4).double()),
                dict(workspace=torch.zeros(8, dtype=torch.uint8), workspace_bytes_=16)):
        with pytest.raises(AssertionError):
            peqa.shared_attention(**{**good, **bad})
