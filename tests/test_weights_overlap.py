"""Strides of the positions' weights that lay two heads' or sequences' weights over each other are refused by both calls that take them."""
import pytest

from test_decode_host import GOOD, cache


@pytest.fixture(scope="module")
def peqa():
    from paper_2305_14152_amd import peqa as p
    p.lib()
    return p


def test_overlaps_are_refused(peqa):
    L = peqa.lib()

    def status(C, ss, hs):
        attend = dict(C=C, rows=1, heads=4, q=GOOD, qs=512, lens=GOOD, seq=GOOD, most=64, window=0, scale=0.1, o=GOOD, os=512, lse=GOOD, w=GOOD, wo=GOOD, ss=ss,
                      hs=hs, ws=None, room=0, stream=None)
        evict = dict(C=C, to=None, n=1, seq=GOOD, lens=GOOD, most=64, w=GOOD, wo=GOOD, ss=ss, hs=hs, keep=30, sinks=4, recent=10, kept=GOOD, new=2 * GOOD, ws=None,
                     room=0, stream=None)
        a, b = L.peqa_paged_attention_weights(*attend.values()), L.peqa_cache_evict(*evict.values())
        assert a == b
        return a

    C = cache(peqa)                                            # 3 sequences, 2 key heads
    # by sequences and by heads, with room between and without (what is refused then is the workspace)
    for ss, hs in ((128, 64), (132, 64), (140, 72), (64, 192), (64, 196), (72, 208)):
        assert status(C, ss, hs) == peqa.PEQA_ERR_WORKSPACE, (ss, hs)
    for ss, hs in ((64, 64), (124, 64), (64, 188), (72, 204), (68, 64), (64, 128)):
        assert status(C, ss, hs) == peqa.PEQA_ERR_SHAPE, (ss, hs)
    # a single one may have any stride that is wide enough
    assert status(cache(peqa, kv_heads=1), 64, 64) == status(cache(peqa, n_seqs=1), 64, 64) == peqa.PEQA_ERR_WORKSPACE
