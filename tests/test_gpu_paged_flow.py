"""The operators on a paged cache together, as a decoding loop uses them: prompts join the pages, drafted trees are rotated, attended and
verified, accepted rows join the pages, eager and from a graph.  The model is one random layer with a head; what it decodes must be what
the same layer decodes without drafts, token by token, from the whole sequence in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_ref as R

pytestmark = pytest.mark.gpu

Hq, Hkv, D, V, PAGE, B = 4, 2, 64, 96, 16, 8
PARENTS = [-1, 0, 0, 1, 1, 2, 3, 6]


class Model:
    def __init__(self):
        g = torch.Generator().manual_seed(41)
        r = lambda *s: torch.randn(*s, generator=g)
        self.embed, self.wq, self.wk, self.wv = r(V, 64), r(64, Hq * D) / 8, r(64, Hkv * D) / 8, r(64, Hkv * D) / 8
        self.head = r(Hq * D, V) * 0.5

    def cuda(self):
        for n in ("embed", "wq", "wk", "wv", "head"):
            setattr(self, n, getattr(self, n).cuda())
        return self

    def project(self, tokens):
        x = self.embed[tokens.long()]
        return (x @ self.wq).unflatten(-1, (Hq, D)), (x @ self.wk).unflatten(-1, (Hkv, D)), (x @ self.wv).unflatten(-1, (Hkv, D))


def greedy_token(m, tokens, w):
    """The token behind a sequence, in 64 bits, and by how much it leads."""
    x = m.embed.double().numpy()[tokens]
    heads = lambda y, h: (x @ y.double().numpy()).reshape(len(tokens), h, D)
    pos = np.arange(len(tokens))
    q, k, v = R.rotate(heads(m.wq, Hq), pos, w, 1.0, False), R.rotate(heads(m.wk, Hkv), pos, w, 1.0, False), heads(m.wv, Hkv)
    out = np.concatenate([R.attention(q[-1:, h], k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)], np.ones((1, len(tokens)), bool), D ** -0.5)[0][0] for h in range(Hq)])
    z = out @ m.head.double().numpy()
    top = np.sort(z)[::-1]
    return int(np.argmax(z)), top[0] - top[1]


@pytest.mark.parametrize("captured", [False, True])
def test_greedy_decoding_with_drafted_trees(captured):
    cpu, m = Model(), Model().cuda()
    table = F.fdd_rope_table(D)
    w, _ = R.frequencies(D, 1e4)
    prompts = [[5, 80, 33, 2, 17], [1], [60] * 3 + list(range(30))]
    N = len(prompts)
    max_pages = 6
    cache = F.fdd_paged_cache(N, N * max_pages, PAGE, max_pages, Hkv, D, dtype=torch.float32)
    cache.page_table.copy_(torch.randperm(N * max_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(N, max_pages))
    # the prompts but for their last token, which is the first root
    P = max(len(p) for p in prompts)
    padded = torch.tensor([p + [0] * (P - len(p)) for p in prompts], dtype=torch.int32, device="cuda")
    held = torch.tensor([len(p) - 1 for p in prompts], dtype=torch.int32, device="cuda")
    _, k, v = m.project(padded)
    F.fdd_paged_append(k.contiguous(), v.contiguous(), cache, table=table, n_rows=held)
    cache.lens.add_(held)
    parents = torch.tensor(PARENTS, dtype=torch.int32, device="cuda")
    tokens = torch.zeros(N, B, dtype=torch.int32, device="cuda")
    mask = torch.empty(N, B, 1, dtype=torch.int64, device="cuda")
    positions = torch.empty(N, B, dtype=torch.int32, device="cuda")
    out = torch.empty(N, B, Hq, D, device="cuda")
    path, emitted = (torch.empty(N, B, dtype=torch.int32, device="cuda") for _ in range(2))
    n_path, chances = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, B, device="cuda")
    wa = torch.empty(max(256, F.fdd_paged_attn_workspace(out, cache, k[:, :B].contiguous().new_empty(N, B, Hkv, D), out.new_empty(N, B, Hkv, D))), dtype=torch.uint8, device="cuda")
    logits = torch.empty(N, B, V, device="cuda")
    wv = torch.empty(F.fdd_tree_verify_workspace(logits), dtype=torch.uint8, device="cuda")
    qs, ks, vs = (torch.empty(N, B, h, D, device="cuda") for h in (Hq, Hkv, Hkv))

    def step():
        F.fdd_tree_mask(parents, lens=cache.lens, mask=mask, positions=positions)
        F.fdd_rope(qs, positions, table, k=ks, out=qs, k_out=ks)
        F.fdd_paged_attn(qs, cache, ks, vs, mask=mask, out=out, workspace=wa)
        torch.matmul(out.view(N * B, Hq * D), m.head, out=logits.view(N * B, V))
        F.fdd_tree_verify(logits, tokens, parents=parents, temperature=0.0, path=path, n_path=n_path, emitted=emitted, chances=chances, workspace=wv)
        F.fdd_paged_append(ks, vs, cache, rows=path, n_rows=n_path)
        cache.lens.add_(n_path)

    graph = None
    if captured:
        keep = cache.lens.clone()
        for _ in range(2):
            for t in (qs, ks, vs):
                t.zero_()
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        cache.lens.copy_(keep)           # (rows behind them are written again before they are used)
    done = [list(p) for p in prompts]
    r = np.random.default_rng(6)
    accepted = 0
    for _ in range(7):
        # trees of guesses, in which the right tokens often come up
        drafts = r.integers(0, V, size=(N, B))
        for n in range(N):
            drafts[n, 0] = done[n][-1]
            sequence = {0: done[n]}
            for i in range(1, B):
                if r.random() < 0.6:
                    drafts[n, i] = greedy_token(cpu, sequence[PARENTS[i]], w)[0]
                sequence[i] = sequence[PARENTS[i]] + [int(drafts[n, i])]
        tokens.copy_(torch.from_numpy(drafts.astype(np.int32)))
        for t, x in zip((qs, ks, vs), m.project(tokens)):
            t.copy_(x)
        if graph is None:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        for n in range(N):
            k_n = int(n_path[n])
            accepted += k_n - 1
            for t in emitted[n, :k_n].tolist():
                right, lead = greedy_token(cpu, done[n], w)
                assert lead > 1e-3, "the test's model has no clear winner here"
                assert t == right
                done[n].append(t)
            assert int(cache.lens[n]) == len(done[n]) - 1
    assert accepted > 10
