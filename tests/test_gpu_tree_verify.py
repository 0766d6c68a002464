"""Verification of drafted tokens on the GPU, against the definition in 64 bits and against the distribution that it stands for."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(np.asarray(x).tolist(), dtype=torch.int32, device="cuda")


def make(dtype, N, B, V, kind, seed, spread=2.0):
    """Logits in which drafted tokens are likely; kind: chain, draft, tree, star, broken."""
    r = np.random.default_rng(seed)
    x = (r.standard_normal((N, B, V)) * spread).astype(np.float32)
    tokens = r.integers(0, V, size=(N, B)).astype(np.int32)
    parents = np.zeros((N, B), dtype=np.int32)
    for i in range(1, B):
        parents[:, i] = {"tree": r.integers(max(0, i - 3), i, size=N), "star": 0, "broken": r.integers(-2, i + 3, size=N)}.get(kind, np.full(N, i - 1))
    draft = None
    if kind == "draft":
        draft = x + r.standard_normal(x.shape).astype(np.float32) * 0.7
        draft = torch.from_numpy(draft).to(DT[dtype])
        d = draft.double().numpy()
        for n in range(N):
            for i in range(B - 1):
                tokens[n, i + 1] = r.choice(V, p=R.softmax(d[n, i], 1.0))
    else:
        for n in range(N):
            for j in range(1, B):
                if 0 <= parents[n, j] < j:
                    x[n, parents[n, j], tokens[n, j]] += np.log(V) + 1.5
    if V > 8:
        x[:, ::2, r.integers(0, V, size=max(1, V // 32))] = -np.inf
    logits = torch.from_numpy(x).to(DT[dtype])
    return logits, draft, tokens, parents, r.random((N, B, 2)).astype(np.float32)


def check(got, logits, draft, tokens, parents, uniforms, counts, temperature, draft_temperature=1.0):
    path, n_path, emitted, chances = (t.cpu().numpy() for t in got)
    N, B, V = logits.shape
    x = logits.double().numpy()
    d = None if draft is None else draft.double().numpy()
    for n in range(N):
        p, e, c = R.verify(x[n], tokens[n], uniforms[n], parents[n], counts[n], temperature, None if d is None else d[n], draft_temperature)
        k = len(p)
        assert n_path[n] == k
        assert path[n].tolist() == p + [-1] * (B - k) and emitted[n].tolist() == e + [-1] * (B - k), n
        # an exponent of up to 2^7 temperatures is off by 3 roundings: 2^-15 of a probability; a chance has two of them
        assert np.all(np.abs(chances[n] - c) <= 2.0 ** -14 * c), n


CASES = [("f32", 1, 1, 5, "chain"), ("bf16", 3, 2, 64, "chain"), ("bf16", 5, 8, 1000, "chain"), ("f32", 4, 9, 4099, "draft"), ("bf16", 6, 5, 777, "draft"), ("f32", 3, 16, 2049, "tree"),
         ("bf16", 8, 32, 9973, "tree"), ("bf16", 2, 40, 513, "star"), ("f32", 3, 33, 100, "star"), ("bf16", 4, 20, 333, "broken"), ("bf16", 1, 3, 152064, "tree"), ("f32", 2, 2, 50001, "draft"),
         ("bf16", 2, 200, 70, "tree"), ("f32", 2, 7, 1, "tree"), ("bf16", 70, 4, 40, "tree"), ("f32", 1, 4, 4100001, "chain")]


@pytest.mark.parametrize("dtype,N,B,V,kind", CASES)
@pytest.mark.parametrize("temperature", [1.0, 0.6, 0.0])
def test_verify(dtype, N, B, V, kind, temperature):
    logits, draft, tokens, parents, u = make(dtype, N, B, V, kind, seed=N * 1000 + B)
    r = np.random.default_rng(1)
    counts = [B] + [int(r.integers(0, B + 1)) for _ in range(N - 1)]
    chain = kind in ("chain", "draft")
    got = F.fdd_tree_verify(logits.cuda(), ints(tokens), torch.from_numpy(u).cuda(), parents=None if chain else ints(parents), draft_logits=None if draft is None else draft.cuda(),
                            n_tokens=ints(counts), temperature=temperature, draft_temperature=1.0)
    check(got, logits, draft if temperature else None, tokens, parents, u, counts, temperature)


def test_draft_temperature_and_tokens_out_of_range():
    logits, draft, tokens, parents, u = make("f32", 6, 6, 300, "draft", seed=3)
    tokens[0, 1], tokens[1, 2], tokens[2, 1] = -1, 300, 1 << 30
    got = F.fdd_tree_verify(logits.cuda(), ints(tokens), torch.from_numpy(u).cuda(), draft_logits=draft.cuda(), temperature=0.8, draft_temperature=1.7)
    check(got, logits, draft, tokens, parents, u, [6] * 6, 0.8, 1.7)
    got = F.fdd_tree_verify(logits.cuda(), ints(tokens), torch.from_numpy(u).cuda(), temperature=0.8)
    check(got, logits, None, tokens, parents, u, [6] * 6, 0.8)


def test_a_token_that_siblings_share_and_drafts_that_account_for_everything():
    V = 16
    logits = torch.full((3, 4, V), -float("inf"))
    logits[0, 0, 3], logits[0, 0, 5] = 0.0, 0.0           # p: 3 and 5; children 3, 3, 5
    logits[1, 0, 7] = 1.0                                 # p: 7 alone, the child that falls with a uniform of nearly 1 is 2
    logits[2, 0, 7] = 1.0
    logits[:, 1:, 1] = 0.0
    tokens = np.array([[0, 3, 3, 5], [0, 2, 2, 2], [0, 7, 7, 7]], dtype=np.int32)
    parents = np.zeros((3, 4), dtype=np.int32)
    for u0 in (0.0, 0.3, 0.6, 0.999):
        u = np.full((3, 4, 2), u0, dtype=np.float32)
        got = F.fdd_tree_verify(logits.cuda(), ints(tokens), torch.from_numpy(u).cuda(), parents=ints(parents))
        check(got, logits, None, tokens, parents, u, [4] * 3, 1.0)
    # the draft is the target: it always stands; where the target has nothing else left, the draw is the target's
    same = torch.randn(2, 3, 50)
    tok = np.array([[0, 4, 9], [0, 1, 2]], dtype=np.int32)
    u = np.full((2, 3, 2), 1 - 2.0 ** -24, dtype=np.float32)
    got = F.fdd_tree_verify(same.cuda(), ints(tok), torch.from_numpy(u).cuda(), draft_logits=same.cuda())
    assert got[1].tolist() == [3, 3]
    other = same.clone()
    other[:, :, 4] = -float("inf")                        # a token the draft could not have drawn, and the target neither
    got = F.fdd_tree_verify(other.cuda(), ints(tok), torch.from_numpy(u * 0.5).cuda(), draft_logits=other.cuda())
    check(got, other, other, tok, np.array([[0, 0, 1]] * 2), u * 0.5, [3, 3], 1.0)


@pytest.mark.parametrize("kind", ["chain", "draft", "star"])
def test_the_first_token_is_distributed_as_the_target(kind):
    V, N = 7, 1 << 15
    r = np.random.default_rng(11)
    target, drafted = r.standard_normal(V) * 1.2, r.standard_normal(V) * 1.2
    p, q = R.softmax(target, 1.0), R.softmax(drafted, 1.0)
    B = 4 if kind == "star" else 2
    logits = torch.tensor(target, dtype=torch.float32, device="cuda").expand(N, B, V).contiguous()
    draft = torch.tensor(drafted, dtype=torch.float32, device="cuda").expand(N, B, V).contiguous() if kind == "draft" else None
    tokens = np.zeros((N, B), dtype=np.int32)
    tokens[:, 1] = r.choice(V, p=q, size=N) if kind == "draft" else 2
    if kind == "star":
        tokens[:, 2], tokens[:, 3] = 5, 2
    u = torch.from_numpy(r.random((N, B, 2)).astype(np.float32)).cuda()
    parents = ints(np.zeros((N, B), dtype=np.int32)) if kind == "star" else None
    _, _, emitted, _ = F.fdd_tree_verify(logits, ints(tokens), u, parents=parents, draft_logits=draft)
    seen = np.bincount(emitted[:, 0].cpu().numpy(), minlength=V) / N
    # five deviations of a count of N draws
    assert np.all(np.abs(seen - p) <= 5 * np.sqrt(p * (1 - p) / N)), (seen, p)


def test_outputs_workspace_stream_and_graph():
    logits, _, tokens, parents, u = make("bf16", 5, 12, 3001, "tree", seed=21)
    x, t, pa = logits.cuda(), ints(tokens), ints(parents)
    uni = torch.from_numpy(u).cuda()
    outs = [torch.full((5, 12), 99, dtype=torch.int32, device="cuda"), torch.full((5,), 99, dtype=torch.int32, device="cuda"), torch.full((5, 12), 99, dtype=torch.int32, device="cuda"),
            torch.full((5, 12), 99.0, device="cuda")]
    ws = torch.empty(F.fdd_tree_verify_workspace(x), dtype=torch.uint8, device="cuda")
    kw = dict(parents=pa, path=outs[0], n_path=outs[1], emitted=outs[2], chances=outs[3], workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    F.fdd_tree_verify(x, t, uni, stream=s, **kw)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        F.fdd_tree_verify(x, t, uni, **kw)
    r = np.random.default_rng(2)
    for _ in range(4):
        u = r.random((5, 12, 2)).astype(np.float32)
        uni.copy_(torch.from_numpy(u))
        for o in outs:
            o.fill_(77)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        check(outs, logits, None, tokens, parents, u, [12] * 5, 1.0)


def test_shared_tree_and_wrong_arguments():
    logits, _, tokens, parents, u = make("f32", 3, 6, 50, "tree", seed=31)
    uni = torch.from_numpy(u).cuda()
    one = F.fdd_tree_verify(logits.cuda(), ints(tokens), uni, parents=ints(parents[0]))
    check(one, logits, None, tokens, np.repeat(parents[:1], 3, 0), u, [6] * 3, 1.0)
    with pytest.raises(TypeError):
        F.fdd_tree_verify(logits.cuda(), ints(tokens), uni[:, :, 0].contiguous())
    with pytest.raises(F.FddError):
        F.fdd_tree_verify(logits.cuda(), ints(tokens), None)
    with pytest.raises(F.FddError):
        F.fdd_tree_verify(logits.cuda(), ints(tokens), uni, parents=ints(parents), draft_logits=logits.cuda())
    with pytest.raises(TypeError):
        F.fdd_tree_verify(logits.cuda(), ints(tokens), uni, draft_logits=logits.cuda().bfloat16())
    greedy = F.fdd_tree_verify(logits.cuda(), ints(tokens), parents=ints(parents), temperature=0.0)
    check(greedy, logits, None, tokens, parents, u, [6] * 3, 0.0)
