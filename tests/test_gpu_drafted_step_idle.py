"""A batch of which one sequence takes no part in a drafted step: it is given no new tokens, its count is cleared, and
its cache and lengths stay as they are, eagerly and in a captured graph."""
import numpy as np
import pytest

from cache_numbers import filled_cache
from test_gpu_drafted_step import B, T, fresh, load

pytestmark = pytest.mark.gpu


def step(ob, c, s, new_lens, active):
    out = ob.draft_attn(c, s["q"], s["k"], s["v"], new_lens=new_lens, out=s["out"], num_splits=3, workspace=s["ws"])
    n_new, tokens = ob.verify_drafts(s["p"], s["pd"], s["drafts"], s["u"], n_new=s["n_new"], tokens=s["tokens"], workspace=s["vws"])
    n_new.mul_(active)
    ob.quantize_append(c, s["k"], s["v"], new_lens=n_new)
    return out, n_new


@pytest.mark.parametrize("idle", [0, 1, 2])
def test_a_sequence_without_a_step(idle):
    import torch
    from paper_2605_19660_amd import binding as ob
    c, d = (filled_cache([120, 255, 500], hq=8, hk=2, pages=6) for _ in range(2))
    s, r = fresh(ob, torch, "bf16"), fresh(ob, torch, "bf16")
    active = torch.ones(B, dtype=torch.int32, device="cuda")
    active[idle] = 0
    new_lens = active * T
    keep = {n: getattr(d, n).clone() for n in ("seq_lens", "res_lens", "res_k", "res_v", "res_norm", "k_codes", "v_codes",
                                               "k_meta", "v_meta", "k_norms")}
    load(torch, r, d, 0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ob, d, r, new_lens, active)
    for n, x in keep.items():
        getattr(d, n).copy_(x)
    before = {n: x.view(B, -1)[idle].clone() for n, x in keep.items() if n.startswith("res")}
    page = c.block_table[idle].long()
    packed = lambda: [getattr(c, n).view(c.num_pages, -1)[page].clone() for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_norms")]
    pages, lens = packed(), c.seq_lens.clone()
    for i in range(8):
        load(torch, s, c, i)
        load(torch, r, d, i)
        out, n_new = step(ob, c, s, new_lens, active)
        graph.replay()
        torch.cuda.synchronize()
        assert not out[idle].any() and int(n_new[idle]) == 0
        assert all(int(out[b].ne(0).any()) and int(n_new[b]) >= 1 for b in range(B) if b != idle)
        lens += n_new
        for x, y in ((out, r["out"]), (n_new, r["n_new"]), (c.seq_lens, d.seq_lens), (c.res_k, d.res_k), (c.k_codes, d.k_codes),
                     (c.seq_lens, lens)):
            assert torch.equal(x, y)
    for n, x in before.items():
        assert torch.equal(getattr(c, n).view(B, -1)[idle], x), n
    assert all(torch.equal(x, y) for x, y in zip(packed(), pages)) and int(c.seq_lens[idle]) == (120, 255, 500)[idle]
