"""Verification where probabilities are small: tokens far below the likeliest one, and what is left of a row behind children that had
nearly all of it."""
import numpy as np
import pytest
import torch

import paper_2605_23163_amd as F
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(np.asarray(x).tolist(), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("depth", [20, 86, 100, 124])
def test_drafted_tokens_far_below_the_likeliest(dtype, depth):
    """Chains whose drafted token has exp(-depth) of the likeliest one's probability, with the target and with the draft: their quotient decides."""
    V, N = 300, 8
    r = np.random.default_rng(depth)
    x, d = (torch.from_numpy(np.minimum(r.standard_normal((N, 2, V)), 2.0).astype(np.float32)) for _ in range(2))
    tokens = np.zeros((N, 2), dtype=np.int32)
    tokens[:, 1] = r.integers(0, V, size=N)
    for n in range(N):      # quotients of about e^-2, e^-1 and above 1
        x[n, 0, tokens[n, 1]], d[n, 0, tokens[n, 1]] = -depth, -depth + (2.0, 1.0, -1.0, -3.0)[n % 4]
    logits, draft = x.to(DT[dtype]), d.to(DT[dtype])
    u = np.full((N, 2, 2), 0.25, dtype=np.float32)
    u[::4], u[4:, :, 0] = 0.5, 0.03
    got = F.fdd_tree_verify(logits.cuda(), ints(tokens), torch.from_numpy(u).cuda(), draft_logits=draft.cuda())
    path, n_path, emitted, chances = (t.cpu().numpy() for t in got)
    for n in range(N):
        p, e, c = R.verify(logits[n].double().numpy(), tokens[n], u[n], [-1, 0], 2, 1.0, draft[n].double().numpy())
        # two probabilities, each off by 2^-16 of itself, and fp32's own half step
        assert np.all(np.abs(chances[n] - c) <= c * (2.0 ** -15 + 2.0 ** -24) * (1 + 2.0 ** -15)), (n, chances[n], c)
        assert n_path[n] == len(p) and emitted[n, :len(e)].tolist() == e, n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [-8, -16, -22])
def test_children_behind_those_that_had_nearly_everything(dtype, left):
    """Two children share all of the row but 2^left of it and fall; the next two are tried with uniforms 2^-9 of themselves beside their borders.

    Both likely entries are the row's largest: their exponentials are 1, and no other entry is within 8 of them (16 bytes and more), so that what is
    left, 1 - 2 / (2 + rest), is off by what the rest is: 2^-16 of itself, and twice that behind the third child, which has a third of it.  A border is
    met to 2^-13 of itself."""
    V, N, B = 5000, 32, 5
    r = np.random.default_rng(-left)
    x = np.full((N, B, V), -np.inf, dtype=np.float32)
    x[:, 1:, 1] = 0.0
    rest = r.standard_normal((N, V - 32)) * 0.5
    tokens = np.zeros((N, B), dtype=np.int32)
    tokens[:, 1:3] = 0, 16
    for n in range(N):
        third, fourth = r.choice(V - 32, size=2, replace=False)
        rest[n, third] = np.log(np.exp(rest[n]).sum() * 0.5)
        rest[n, fourth] = np.log(np.exp(rest[n]).sum() * 0.3)
        tokens[n, 3:] = third + 32, fourth + 32
        x[n, 0, 32:] = rest[n] + left * np.log(2.0) - np.log(np.exp(rest[n]).sum()) + np.log(2.0)
        x[n, 0, [0, 16]] = 0.0
    logits = torch.from_numpy(x).to(DT[dtype])
    parents = np.zeros((N, B), dtype=np.int32)
    u = r.random((N, B, 2)).astype(np.float32)
    u[:, 1:3, 0] = 1 - 2.0 ** -24
    want_path = []
    for n in range(N):
        e = np.exp(logits[n, 0].double().numpy())
        e[[0, 16]] = 0.0
        w3, w4, W = e[tokens[n, 3]], e[tokens[n, 4]], e.sum()
        third = w3 / W * (1 + (2.0 ** -9 if n & 1 else -2.0 ** -9))
        fourth = w4 / (W - w3) * (1 + (2.0 ** -9 if n & 2 else -2.0 ** -9))
        u[n, 3:, 0] = third, fourth
        want_path.append([0] if n & 3 == 3 else [0, 4] if n & 1 else [0, 3])
    path, n_path, emitted, _ = (t.cpu().numpy() for t in F.fdd_tree_verify(logits.cuda(), ints(tokens), torch.from_numpy(u).cuda(), parents=ints(parents)))
    wrong = [n for n in range(N) if path[n, :n_path[n]].tolist() != want_path[n]]
    assert not wrong, [(n, path[n].tolist(), want_path[n]) for n in wrong]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_in_rising_order(dtype):
    """Every entry is larger than those before it: the sum's reference moves as often as it can."""
    V, B = 200000, 3
    x = torch.arange(V, dtype=torch.float64).mul(60.0 / V).expand(1, B, V).to(DT[dtype]).contiguous()
    tokens = np.array([[0, V - 1, 120000]], dtype=np.int32)
    parents = np.zeros((1, B), dtype=np.int32)
    u = np.full((1, B, 2), 0.9, dtype=np.float32)
    got = F.fdd_tree_verify(x.cuda(), ints(tokens), torch.from_numpy(u).cuda(), parents=ints(parents))
    p, e, c = R.verify(x[0].double().numpy(), tokens[0], u[0], parents[0], B, 1.0)
    assert np.all(np.abs(got[3].cpu().numpy()[0] - c) <= c * (2.0 ** -16 + 2.0 ** -24) * (1 + 2.0 ** -16))
    assert got[0].tolist()[0][:len(p)] == p and got[2].tolist()[0][:len(e)] == e
