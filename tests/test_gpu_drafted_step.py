"""A decoding step with drafted tokens as a program makes it: positions, attention, verification, the append of what
stands, and the history read back; eagerly and as one captured graph, over steps that cross page ends."""
import numpy as np
import pytest

from cache_numbers import filled_cache, torch_type
from test_gpu_draft import attention
from test_gpu_verify import rows, rule

pytestmark = pytest.mark.gpu

B, T, HQ, HK, V = 3, 5, 8, 2, 997


def step(ob, c, s):
    """Last token and T - 1 drafts of every sequence; returns the outputs, the counts and the tokens."""
    ob.rope(s["q"], s["k"], s["pos"], s["inv"], axes=s["axes"], out_q=s["qr"], out_k=s["kr"])
    out = ob.draft_attn(c, s["qr"], s["kr"], s["v"], out=s["out"], max_seq_len_hint=2000, num_splits=3, workspace=s["ws"])
    n_new, tokens = ob.verify_drafts(s["p"], s["pd"], s["drafts"], s["u"], n_new=s["n_new"], tokens=s["tokens"], workspace=s["vws"])
    ob.quantize_append(c, s["kr"], s["v"], new_lens=n_new)
    return out, n_new, tokens


def fresh(ob, torch, io):
    e = lambda *shape, dtype=torch_type(io): torch.zeros(*shape, dtype=dtype, device="cuda")
    cfg = ob.Config(HQ, HK)
    s = {"q": e(B, T, HQ, 128), "k": e(B, T, HK, 128), "v": e(B, T, HK, 128), "pos": e(3, B * T, dtype=torch.int32),
         "inv": torch.from_numpy((1e4 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)).cuda(),
         "axes": ob.rope_axes([24, 20, 20], interleaved=True), "p": e(B, T, V, dtype=torch.float32),
         "pd": e(B, T - 1, V, dtype=torch.float32), "drafts": e(B, T - 1, dtype=torch.int32), "u": e(B, T, dtype=torch.float32),
         "n_new": e(B, dtype=torch.int32), "tokens": e(B, T, dtype=torch.int32),
         "ws": e(ob.draft_workspace_bytes(cfg, B, T, 3), dtype=torch.uint8), "vws": e(ob.verify_workspace_bytes(B, V), dtype=torch.uint8)}
    s["qr"], s["kr"], s["out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"]), torch.zeros_like(s["q"])
    return s


def load(torch, s, c, seed):
    g = torch.Generator().manual_seed(seed)
    for n in ("q", "k", "v"):
        s[n].copy_(torch.randn(s[n].shape, generator=g))
    at = c.seq_lens[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
    s["pos"].copy_(at.view(1, -1).expand(3, -1) // torch.tensor([[1], [4], [7]], device="cuda"))
    p, pd, drafts, u = rows(B, T - 1, V, "f32", seed, near=0.4)
    for n, x in (("p", p), ("pd", pd), ("drafts", drafts), ("u", u)):
        s[n].copy_(x)


@pytest.mark.parametrize("io", ["bf16", "f16"])
def test_steps_of_a_server(io):
    import torch
    from paper_2605_19660_amd import binding as ob
    a, b = (filled_cache([120, 255, 500], hq=HQ, hk=HK, io=io, pages=6, scattered=True) for _ in range(2))
    s, r = fresh(ob, torch, io), fresh(ob, torch, io)
    load(torch, r, b, 0)
    keep = {n: getattr(b, n).clone() for n in ("seq_lens", "res_lens", "res_k", "res_v", "res_norm", "k_codes", "k_meta",
                                               "k_norms", "v_codes", "v_meta")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ob, b, r)
    for n, x in keep.items():
        getattr(b, n).copy_(x)
    total = a.seq_lens.clone()
    for i in range(12):
        load(torch, s, a, i)
        load(torch, r, b, i)
        want = None
        if i % 4 == 0:
            qr, kr = ob.rope(s["q"], s["k"], s["pos"], s["inv"], axes=s["axes"])
            want = attention(a, *(x.double().cpu().numpy() for x in (qr, kr, s["v"])), None, io)
        out, n_new, tokens = step(ob, a, s)
        if want is not None:
            assert (np.abs(out.double().cpu().numpy() - want[0]) <= want[1]).all()
        n, t = rule(*(s[x].double().cpu().numpy() for x in ("p", "pd")), s["drafts"].cpu().numpy(), s["u"].cpu().numpy(), None)
        assert np.array_equal(n_new.cpu().numpy(), n) and np.array_equal(tokens.cpu().numpy(), t)
        total += n_new
        assert torch.equal(a.seq_lens, total)
        # the keys of what stood, back out of the window: normalised to fp16 and multiplied by the fp16 norm there,
        # so each channel is off by half a step of both and of the last rounding, of the vector's length at most
        # (where the step went past a block's end its first tokens are in a page by now, quantized)
        back = torch.zeros(B, T, HK, 128, device="cuda")
        ob.cache_read(a, total - n_new, k=back)
        in_window = torch.minimum(n_new, a.res_lens).tolist()
        for q in range(B):
            k, got = s["kr"][q, n[q] - in_window[q]:n[q]].float(), back[q, n[q] - in_window[q]:n[q]]
            assert float(((got - k).norm(dim=-1) / k.norm(dim=-1)).max()) <= 2 * 2.0 ** -11 + 1e-6
            assert not back[q, n[q]:].any()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((out, r["out"]), (n_new, r["n_new"]), (tokens, r["tokens"]), (a.seq_lens, b.seq_lens), (a.res_lens, b.res_lens),
                     (a.k_codes, b.k_codes), (a.v_codes, b.v_codes), (a.res_k, b.res_k)):
            assert torch.equal(x, y)
    assert int((total - torch.tensor([120, 255, 500], device="cuda")).min()) > 12
