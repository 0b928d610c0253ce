"""A serving step as a program makes it: plan, positions, append, attention and the draw, for two layers that share
lengths and a block table; eagerly and as one captured graph, over steps in which requests come, grow, draft and end."""
import numpy as np
import pytest

from q8_numbers import stands_for

pytestmark = pytest.mark.gpu

B, P, PAGES, HQ, HK, V, ROWS, LAYERS, MAX_NEW = 5, 6, 18, 8, 2, 1003, 260, 2, 200


class Server:
    """The buffers of a step and two layers' caches."""

    def __init__(self, ob, torch, io):
        e = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype, device="cuda")
        self.ob, self.io, t = ob, io, ob.torch_dtype(io)
        self.lens, self.keep, self.want, self.n_free = e(B), e(B), e(B), e(1)
        self.table, self.free = e(B, P), e(PAGES)
        self.out = dict(new_lens=e(B), row_starts=e(B + 1), positions=e(ROWS), row_seq=e(ROWS), slots=e(ROWS))
        self.layers = [ob.Q8Cache(HK, B, P, block=32, io_dtype=io, num_pages=PAGES, block_table=self.table) for _ in range(LAYERS)]
        self.qkv = e(LAYERS, ROWS, (HQ + 2 * HK) * 128, dtype=t)
        self.q, self.k = e(LAYERS, ROWS, HQ, 128, dtype=t), e(LAYERS, ROWS, HK, 128, dtype=t)
        self.o = e(LAYERS, ROWS, HQ, 128, dtype=t)
        self.inv = torch.from_numpy((1e4 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)).cuda()
        self.logits, self.u = e(B, V, dtype=torch.float32), e(B, dtype=torch.float32)
        self.k_top, self.p_top = e(B), torch.full((B,), 0.9, device="cuda")
        self.k_top += torch.tensor([0, 40, 1, 0, 2000], dtype=torch.int32, device="cuda")
        self.tokens, self.probs = e(B), e(B, V, dtype=torch.float32)
        self.ws = e(ob.q8_workspace_bytes(self.layers[0], HQ, MAX_NEW, 2), dtype=torch.uint8)
        self.sample_ws = e(ob.sample_workspace_bytes(B, V), dtype=torch.uint8)
        self.reset(torch)

    def reset(self, torch):
        for x in (self.lens, self.keep, self.want, self.table):
            x.zero_()
        self.free.copy_(torch.arange(PAGES))
        self.n_free.fill_(PAGES)
        for c in self.layers:
            for x in (c.k_codes, c.v_codes, c.k_scales, c.v_scales, c.win_k, c.win_v):
                x.zero_()

    def step(self):
        ob = self.ob
        p = ob.plan_step(self.lens, self.want, self.table, self.free, self.n_free, ROWS, keep=self.keep, lens_out=self.lens,
                         n_free_out=self.n_free, **self.out)
        for l, c in enumerate(self.layers):
            q, k, v = (self.qkv[l][:, a * 128:b * 128].unflatten(1, (b - a, 128)) for a, b in ((0, HQ), (HQ, HQ + HK), (HQ + HK, HQ + 2 * HK)))
            ob.rope(q, k, p.positions, self.inv, out_q=self.q[l], out_k=self.k[l])
            ob.q8_append(c, self.k[l], v, p.lens, new_lens=p.new_lens, row_starts=p.row_starts, max_new=MAX_NEW)
            ob.q8_attn(c, self.q[l], p.lens, new_lens=p.new_lens, row_starts=p.row_starts, max_new=MAX_NEW, out=self.o[l], num_splits=2,
                       workspace=self.ws)
        ob.sample(self.logits, self.u, top_k=self.k_top, top_p=self.p_top, tokens=self.tokens, probs=self.probs,
                  workspace=self.sample_ws)


def wishes(rng, lens, i):
    """What every sequence keeps and wants: drafts taken back, prompts, ends with another request in their place."""
    keep, want = lens.copy(), np.ones(B, int)
    for b in range(B):
        r = rng.random()
        if lens[b] == 0 or r < 0.1:
            keep[b], want[b] = 0, rng.integers(1, MAX_NEW)
        elif r < 0.4:
            keep[b], want[b] = max(lens[b] - rng.integers(0, 4), 1), 4
        elif r < 0.5:
            want[b] = 0
        elif r < 0.6:
            want[b] = rng.integers(1, MAX_NEW)
    return keep, want


@pytest.mark.parametrize("io", ["bf16", "f16"])
def test_steps_of_a_server(io):
    import torch
    from paper_2605_19660_amd import binding as ob
    code = {"bf16": ob.BF16, "f16": ob.F16}[io]
    a, r = Server(ob, torch, code), Server(ob, torch, code)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.step()
    r.reset(torch)
    history = [[[None, None] for _ in range(B)] for _ in range(LAYERS)]    # keys and values of every sequence, as rope made them
    rng, waited = np.random.default_rng(0), 0
    for i in range(30):
        lens = a.lens.cpu().numpy().astype(int)
        keep, want = wishes(rng, lens, i)
        g = torch.Generator().manual_seed(i)
        qkv = torch.randn(a.qkv.shape, generator=g)
        logits = torch.randn(a.logits.shape, generator=g) * 3
        u = torch.rand(B, generator=g)
        for s in (a, r):
            s.keep.copy_(torch.from_numpy(keep)), s.want.copy_(torch.from_numpy(want))
            s.qkv.copy_(qkv), s.logits.copy_(logits), s.u.copy_(u)
            s.o.fill_(7.0)
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        n, starts, new = a.lens.cpu().numpy(), a.out["row_starts"].cpu().numpy(), a.out["new_lens"].cpu().numpy()
        waited += int((new < want).sum())
        assert (n == keep + new).all()
        for l in range(LAYERS):
            qkv_l, kl, ql = (x[l].double().cpu().numpy() for x in (a.qkv, a.k, a.q))
            vl = qkv_l[:, (HQ + HK) * 128:].reshape(ROWS, HK, 128)
            for b in range(B):
                rows = slice(starts[b], starts[b] + new[b])
                for j, x in enumerate((kl, vl)):
                    old = history[l][b][j]
                    old = np.zeros((0, HK, 128)) if old is None else old[:keep[b]]
                    history[l][b][j] = np.concatenate([old, x[rows]])
                if i % 5 == 0 and l == i // 5 % LAYERS:
                    got = a.o[l].double().cpu().numpy()[rows]
                    for h in range(HQ):
                        k, v = (stands_for(history[l][b][j][:, h // 4], 32, io)[0] for j in (0, 1))
                        for t in range(new[b]):
                            end = keep[b] + t + 1
                            x = k[:end] @ ql[starts[b] + t, h] / np.sqrt(128)
                            p = np.exp(x - x.max())
                            o = (p @ v[:end]) / p.sum()
                            # half a step of the output, and 2^-15 of the weights (logits of about 10 off by 2^-17 a
                            # unit in fp32, two limbs of 2^-17)
                            tol = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[io] * np.abs(o) + 2.0 ** -13 * (p @ np.abs(v[:end])) / p.sum() + 2.0 ** -24
                            assert (np.abs(got[t, h] - o) <= tol).all(), (i, l, b, h, t)
            assert (a.o[l][int(starts[B]):] == 7.0).all()
        same = [(getattr(a, x), getattr(r, x)) for x in ("lens", "table", "free", "n_free", "o", "tokens", "probs")]
        same += [(a.out[x], r.out[x]) for x in a.out]
        same += [(getattr(c, x), getattr(d, x)) for c, d in zip(a.layers, r.layers) for x in ("k_codes", "v_codes", "k_scales", "v_scales", "win_k", "win_v")]
        for j, (x, y) in enumerate(same):
            assert torch.equal(x, y), (i, j)
        assert (a.probs.sum(-1) - 1).abs().max() < 1e-5 and (a.probs.gather(1, a.tokens.long()[:, None]) > 0).all()
    assert waited > 0       # (the pages ran short at times)


def test_the_draw_and_the_check_of_drafts():
    """Drafts drawn by one row of probabilities, checked against another: the distribution that sample gives is what
    verify_drafts reads, and drafts that were drawn from the target itself all stand."""
    import torch
    from paper_2605_19660_amd import binding as ob
    g = torch.Generator().manual_seed(1)
    B, T, V = 6, 4, 3001
    logits = (torch.randn(B, T + 1, V, generator=g) * 3).cuda()
    u, w = torch.rand(B * (T + 1), generator=g).cuda(), torch.rand(B, T + 1, generator=g).cuda()
    p = torch.full((B * (T + 1),), 0.8, device="cuda")
    tokens, probs = ob.sample(logits.view(-1, V), u, top_p=p, probs=True)
    target = probs.view(B, T + 1, V)
    drafts = tokens.view(B, T + 1)[:, :T].contiguous()
    n_new, out = ob.verify_drafts(target, target[:, :T].contiguous(), drafts, w)
    assert (n_new == T + 1).all() and torch.equal(out[:, :T], drafts)
    again, _ = ob.sample(logits[:, T], w[:, T].contiguous(), top_p=p[:B])
    # (the same running sums, of probabilities rounded to fp32: another token only where u meets a border)
    assert int((again != out[:, T]).sum()) <= 1
