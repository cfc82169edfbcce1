"""Host side of the norms with the rotation: sizes and refusals, all before a device is touched."""
import pytest

from test_decode_host import BAD, GOOD, ODD, cache


@pytest.fixture(scope="module")
def peqa():
    from paper_2305_14152_amd import peqa as p
    p.lib()
    return p


def test_append_refusals(peqa):
    L, C = peqa.lib(), cache(peqa)

    def call(**changes):
        d = dict(C=C, T=3, pos=GOOD, place=None, seq=None, cos=GOOD, sin=GOOD, n_pos=64, rot=128, il=0, wq=GOOD, wk=GOOD, eps=1e-6, heads=4, q=GOOD,
                 qs=512, k=GOOD, ks=256, v=GOOD, vs=256, o=GOOD, os=512, stream=None)
        d.update(changes)
        return L.peqa_norm_rope_append(*d.values())

    for bad, status in [(dict(C=None), 1), (dict(C=cache(peqa, head_dim=100)), 2), (dict(pos=None), 1), (dict(k=None), 1), (dict(v=None), 1),
                        (dict(q=None), 1), (dict(o=None), 1), (dict(cos=None), 1), (dict(T=0), 2), (dict(T=4), 2), (dict(rot=24), 8), (dict(qs=504), 2),
                        (dict(eps=0.0), 8), (dict(eps=-1e-6), 8), (dict(eps=float("nan")), 8), (dict(eps=float("inf")), 8), (dict(wq=BAD), 5),
                        (dict(wk=BAD), 5), (dict(place=ODD), 5), (dict(q=BAD), 5), (dict(os=516), 5)]:
        assert call(**bad) == status, bad


def test_training_refusals_and_sizes(peqa):
    L = peqa.lib()

    def forward(**changes):
        d = dict(T=3, pos=GOOD, cos=GOOD, sin=GOOD, n_pos=64, rot=128, il=0, wq=GOOD, wk=GOOD, eps=1e-6, dim=128, heads=4, kv=2, q=GOOD, qs=512, k=GOOD,
                 ks=256, qo=GOOD, qos=512, ko=GOOD, kos=256, stream=None)
        d.update(changes)
        return L.peqa_norm_rope(*d.values())

    def backward(**changes):
        d = dict(T=3, pos=GOOD, cos=GOOD, sin=GOOD, n_pos=64, rot=128, il=0, wq=GOOD, wk=GOOD, eps=1e-6, dim=128, heads=4, kv=2, q=GOOD, qs=512, k=GOOD,
                 ks=256, qo=GOOD, qos=512, ko=GOOD, kos=256, dq=GOOD, dqs=512, dk=GOOD, dks=256, dwq=GOOD, dwk=GOOD, ws=GOOD, room=1 << 20,
                 stream=None)
        d.update(changes)
        return L.peqa_norm_rope_bwd(*d.values())

    both = [(dict(T=0), 2), (dict(T=2 ** 31 - 1), 2), (dict(dim=96), 2), (dict(heads=0), 2), (dict(kv=0), 2), (dict(heads=65537), 2), (dict(pos=None), 1),
            (dict(q=None), 1), (dict(k=None), 1), (dict(qo=None), 1), (dict(ko=None), 1), (dict(rot=144), 8), (dict(rot=24), 8), (dict(rot=-16), 8),
            (dict(n_pos=0), 8), (dict(eps=0.0), 8), (dict(eps=float("nan")), 8), (dict(cos=None), 1), (dict(sin=None), 1), (dict(qs=504), 2),
            (dict(ks=248), 2), (dict(qos=504), 2), (dict(kos=248), 2), (dict(q=BAD), 5), (dict(k=BAD), 5), (dict(qo=BAD), 5), (dict(ko=BAD), 5),
            (dict(wq=BAD), 5), (dict(wk=BAD), 5), (dict(qs=516), 5), (dict(kos=260), 5), (dict(cos=BAD), 5), (dict(sin=BAD), 5), (dict(pos=ODD), 5)]
    for bad, status in both:
        assert forward(**bad) == status, bad
        assert backward(**bad) == status, bad
    need = peqa.norm_rope_bwd_workspace_bytes(3, 4, 2, 128)
    for bad, status in [(dict(dq=None), 1), (dict(dk=None), 1), (dict(dqs=504), 2), (dict(dks=248), 2), (dict(dq=BAD), 5), (dict(dks=260), 5),
                        (dict(dwq=BAD), 5), (dict(dwk=BAD), 5), (dict(ws=None), 6), (dict(room=need - 1), 6), (dict(ws=BAD), 5)]:
        assert backward(**bad) == status, bad
    assert peqa.norm_rope_bwd_workspace_bytes(0, 4, 2, 128) == 0 and peqa.norm_rope_bwd_workspace_bytes(3, 4, 2, 80) == 0
    assert peqa.norm_rope_bwd_workspace_bytes(1 << 16, 64, 64, 256) <= 2 << 20


def test_binding(peqa):
    import torch
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    c = peqa.kv_cache(k, k.clone(), torch.zeros((3, 4), dtype=torch.int32))
    bf16 = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)  # noqa: E731
    pos, cos, w = torch.zeros(3, dtype=torch.int32), torch.zeros(64, 64), torch.ones(128)
    q, k, v = bf16(3, 4, 128), bf16(3, 2, 128), bf16(3, 2, 128)
    good = dict(cache=c, q=q, k=k, v=v, pos=pos, cos=cos, sin=cos, q_weight=w, k_weight=w, eps=1e-6, q_out=q.clone(), place=pos, seq=pos, stream=0)
    for bad in (dict(place=pos.long()), dict(place=pos[:2]), dict(pos=pos.float()), dict(q_weight=w.double()), dict(k_weight=w[:64]),
                dict(q_weight=w.bfloat16()), dict(q=q.half()), dict(q=q.transpose(0, 1)), dict(v=bf16(3, 4, 128)), dict(q_out=bf16(3, 4, 64)),
                dict(sin=torch.zeros(64, 32)), dict(cos=cos.double())):
        with pytest.raises(AssertionError):
            peqa.norm_rope_append(**{**good, **bad})
    with pytest.raises(peqa.PeqaError) as e:
        peqa.norm_rope_append(**{**good, "eps": 0.0})
    assert e.value.status == peqa.PEQA_ERR_PARAM
    good = dict(q=q, k=k, pos=pos, cos=cos, sin=cos, q_weight=w, k_weight=w, eps=1e-6, stream=0)
    outs = dict(q_out=q.clone(), k_out=k.clone())
    grads = dict(d_q_out=q.clone(), d_k_out=k.clone(), dq=q.clone(), dk=k.clone(), d_q_weight=w.clone(), d_k_weight=w.clone(), workspace=None,
                 workspace_bytes_=0)
    both = (dict(pos=pos.long()), dict(q_weight=w.double()), dict(k_weight=w[:64]), dict(q=q.half()), dict(k=bf16(4, 2, 128)), dict(k=bf16(3, 2, 64)))
    for bad in both + (dict(q_out=bf16(3, 2, 128)), dict(k_out=bf16(2, 2, 128)), dict(q_out=q.float())):
        with pytest.raises(AssertionError):
            peqa.norm_rope(**{**good, **outs, **bad})
    for bad in both + (dict(dq=bf16(3, 2, 128)), dict(d_k_out=k.float()), dict(d_q_weight=w[:100]), dict(d_k_weight=w.half()),
                       dict(workspace=torch.zeros(8, dtype=torch.uint8), workspace_bytes_=16)):
        with pytest.raises(AssertionError):
            peqa.norm_rope_bwd(**{**good, **grads, **bad})
    with pytest.raises(peqa.PeqaError) as e:
        peqa.norm_rope_bwd(**{**good, **grads})
    assert e.value.status == peqa.PEQA_ERR_WORKSPACE
