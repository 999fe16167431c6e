"""The paged decoder (serving.py) through a life of sequences -- prompts, steps, forks, releases, compaction -- against attention in 64 bits over the
rows that were given, with the codes' error as the only liberty: outputs are compared with those over what the cache holds (read back), and what it
holds with what was given."""
import numpy as np
import pytest
import torch

from paper_2408_01890_b200 import binding as lb
from paper_2408_01890_b200 import serving
from paged_reference import shared_scores, softmax_v

pytestmark = pytest.mark.gpu
STD, SH = lb.CACHE_STANDARD, lb.CACHE_SHARED


@pytest.mark.parametrize("dtype,P,Hkv", [(lb.S8, 16, 8), (lb.E4M3, 32, 32)])
def test_a_decoders_life(dtype, P, Hkv):
    B, Hq, d, r, m = 5, 32, 128, 21, 64
    kinds = [STD, SH, SH, STD, SH]
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    weights = [None if k == STD else ((torch.randn((Hq, m), generator=g, device="cuda") * Hq ** -0.5).bfloat16(),
                                      (torch.randn((m, Hq), generator=g, device="cuda") * m ** -0.5).bfloat16()) for k in kinds]
    dec = serving.PagedDecoder(kinds, weights, rows=B, n_pages=60, max_len=128, Hq=Hq, Hkv=Hkv, d=d, r=r, page_tokens=P, dtype=dtype)
    counts = torch.tensor([33, 0, 16, 1, 70], dtype=torch.int32, device="cuda")
    prompt = serving._tokens(kinds, B, 70, Hq, Hkv, d, r, g)
    dec.admit([t[1:] for t in prompt], counts)
    given = [[[(prompt[l][1][b, :n], prompt[l][2][b, :n])] for b, n in enumerate(counts.tolist())] for l in range(len(kinds))]   # [layer][row]: rows so far
    outs = [torch.empty((B, 1, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in kinds]

    def step():
        token = serving._tokens(kinds, B, 1, Hq, Hkv, d, r, g)
        live = (dec.lens > 0).tolist()
        dec.step(token, outs)
        assert lb.lisa_check() == lb.OK
        lens = dec.lens.tolist()
        for l, kind in enumerate(kinds):
            for b in range(B):
                if live[b]:
                    given[l][b] = given[l][b] + [(token[l][1][b], token[l][2][b])]
        for b in range(B):
            if not live[b]:
                assert lens[b] == 0 and all((o[b] == 0).all() for o in outs)
                continue
            a = None
            for l, kind in enumerate(kinds):
                n = lens[b]
                k = torch.empty((B, n, Hkv, r if kind == SH else d), device="cuda")
                v = torch.empty((B, n, Hkv, d), device="cuda")
                lb.lisa_paged_read(dec.cache.layers[l], dec.pages.table, None, k, v, dec.lens)
                want = [torch.cat([x[i] for x in given[l][b]]).float() for i in (0, 1)]
                for have, w in ((k[b], want[0]), (v[b], want[1])):      # half a unit of a block's scale, and as much for a rescaling
                    assert w.shape == have.shape and (have - w).abs().max() < 5.0 * (2 / 127 if dtype == lb.S8 else 2 / 16)
                K, V = k[b].double().cpu().numpy().transpose(1, 0, 2), v[b].double().cpu().numpy().transpose(1, 0, 2)
                q = token[l][0][b, 0].double().cpu().numpy()
                if kind == STD:
                    a = np.einsum("hd,hnd->hn", q, np.repeat(K, Hq // Hkv, 0)) / np.sqrt(d)
                else:
                    a = shared_scores(a, q, K, lb.Link(token[l][0], None, *weights[l], act=lb.ACT_RELU))
                ref = softmax_v(a, V, Hq // Hkv)
                got = outs[l][b, 0].double().cpu().numpy()
                assert np.abs(got - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 1e-4, (b, l)

    step()
    step()
    parent = [4, 0, 2, -1, 4]                                           # row 4 branches, row 0 moves to the idle slot, row 3 ends
    dec.fork(torch.tensor(parent, dtype=torch.int32, device="cuda"))
    given = [[layer[q] if q >= 0 else [] for q in parent] for layer in given]
    step()
    dec.release([2])
    for layer in given:
        layer[2] = []
    dec.compact()
    used = int((dec.pages.refs > 0).sum())
    assert bool((dec.pages.refs[:used] > 0).all()) and int(dec.pages.table.max()) == used - 1
    step()
    # a sequence comes to a freed row
    counts = torch.tensor([0, 0, 40, 0, 0], dtype=torch.int32, device="cuda")
    prompt = serving._tokens(kinds, B, 40, Hq, Hkv, d, r, g)
    dec.admit([t[1:] for t in prompt], counts)
    for l in range(len(kinds)):
        given[l][2] = [(prompt[l][1][2], prompt[l][2][2])]
    step()


def test_the_example_runs(capsys):
    serving.main()
    assert "us a step" in capsys.readouterr().out
