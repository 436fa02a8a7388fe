"""GPU tests of the verification where cancellation takes digits: what is left of a distribution after several rejections, and
the difference of a target and a draft that nearly agree.  The oracle computes in double precision; results have to be equal."""
import numpy as np
import pytest
import torch

from oracle import tree as ot

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_08097_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def verify(L, logits, tokens, parent, u, temp, draft=None):
    B, T, V = logits.shape
    i32 = lambda v: torch.tensor(np.asarray(v).tolist(), dtype=torch.int32, device="cuda")  # noqa: E731
    path, n, nxt = i32(np.full((B, T), 99)), i32([99] * B), i32([99] * B)
    L.verify_tree(logits, i32(tokens), i32(parent), i32([T] * B), torch.tensor(u, dtype=torch.float32, device="cuda"),
                  torch.full((B,), temp, device="cuda"), path, n, nxt, draft_probs=draft)
    torch.cuda.synchronize()
    ref = ot.verify_tree(logits.double().cpu().numpy(), tokens, parent, [T] * B, np.asarray(u, np.float32), np.full(B, temp, np.float32), T,
                         None if draft is None else draft.double().cpu().numpy())
    return [t.cpu().numpy() for t in (path, n, nxt)], ref


def test_the_last_tokens_after_rejections_that_took_nearly_everything(L):
    """Four tokens, each about 2^-24 of the one before, all drafted; random numbers at their largest reject the first three.  The
    last one is then all that is left, and is kept whatever the random number is."""
    rng = np.random.default_rng(0)
    N, T, V = 64, 5, 64
    x, tokens = np.full((N, T, V), -np.inf, np.float32), np.zeros((N, T), np.int32)
    parent, u = np.tile([-1, 0, 0, 0, 0], (N, 1)).astype(np.int32), np.full((N, T), 1 - 2.0 ** -24, np.float32)
    u[:, 0] = 0.5
    for i in range(N):
        t = rng.choice(V, 4, replace=False)
        x[i, :, t[0]] = 0.0
        for k, step in enumerate((rng.uniform(15.6, 16.6), rng.uniform(15.0, 16.6), rng.uniform(14.0, 16.6))):
            x[i, :, t[k + 1]] = x[i, 0, t[k]] - step
        tokens[i, 1:] = t
    got, ref = verify(L, torch.tensor(x, device="cuda"), tokens, parent, u, 1.0)
    assert (ref[0][:, 1] == 4).all()
    assert all(np.array_equal(g, r) for g, r in zip(got, ref)), (got[0][:, 1], got[2] - ref[2])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_draft_that_differs_from_the_target_in_the_last_bits(L, dtype):
    """The draft is the target rounded to fp32, all but the drafted token, which is rejected: the next token is drawn from the
    differences, about 2^-25 of either.  (A weight that is off by e moves the border between two tokens by e 2^25 or so of a
    token's share: 1e-13 by 3e-6 of it, once in 1e5 draws; 2e-10 by more than a hundredth.)"""
    rng = np.random.default_rng(1)
    N, V = 512, 2000
    x = torch.tensor(rng.standard_normal((N, 2, V)), device="cuda").to(dtype)
    p = torch.softmax(x.double() / 0.9000000357627869, -1)                # (the temperature as fp32 holds it)
    q = p.float()
    tokens, parent = rng.integers(0, V, (N, 2)).astype(np.int32), np.tile([-1, 0], (N, 1)).astype(np.int32)
    q[torch.arange(N), 0, torch.tensor(tokens[:, 1].astype(np.int64))] = 0.9
    u = rng.random((N, 2)).astype(np.float32)
    u[:, 1] = 1 - 2.0 ** -24
    got, ref = verify(L, x, tokens, parent, u, 0.9, q)
    assert (ref[1] == 1).all()
    assert all(np.array_equal(g, r) for g, r in zip(got, ref)), int((got[2] != ref[2]).sum())


@pytest.mark.parametrize("draft", [False, True], ids=["fixed", "drawn"])
def test_tokens_far_below_the_likeliest(L, draft):
    """Shares from e^-240 to e^-590 of the largest still count: a random number of 0 keeps such a child, and where the draft
    takes all of the likely token, the unlikely ones share what is left."""
    rng = np.random.default_rng(2)
    N, V = 96, 40
    x = np.full((N, 2, V), -np.inf, np.float32)
    tokens, parent, u = np.zeros((N, 2), np.int32), np.tile([-1, 0], (N, 1)).astype(np.int32), np.zeros((N, 2), np.float32)
    q = np.zeros((N, 2, V), np.float32)
    for i in range(N):
        t = rng.choice(V, 6, replace=False)
        x[i, :, t[0]] = 7.0
        x[i, :, t[1:]] = (7.0 - 0.5 * rng.uniform(240 + 3 * i, 245 + 3 * i, (5, 1)))      # (240 to 530 temperatures of 0.5 below)
        q[i, :, t[0]] = 1.0
        tokens[i, 1] = t[1 + i % 5]
        if draft:                                         # rejected: it has a share of the draft, and none of the target's
            tokens[i, 1] = rng.choice(np.setdiff1d(np.arange(V), t))
            q[i, :, tokens[i, 1]] = 0.25
            u[i] = rng.random(2)
    got, ref = verify(L, torch.tensor(x, device="cuda"), tokens, parent, u, 0.5, torch.tensor(q, device="cuda") if draft else None)
    assert (ref[1] == (1 if draft else 2)).all()
    assert all(np.array_equal(g, r) for g, r in zip(got, ref)), int((got[2] != ref[2]).sum())


def test_several_rejections_that_leave_only_tokens_the_draft_has_not(L):
    """The draft takes all of the likely token and more than the target has of the second; five tokens at e^-60 to e^-300 are
    left after the first rejection, and share everything after the others too."""
    rng = np.random.default_rng(3)
    N, T, V = 128, 5, 40
    x, q = np.full((N, T, V), -np.inf, np.float32), np.zeros((N, T, V), np.float32)
    tokens, parent = np.zeros((N, T), np.int32), np.tile([-1, 0, 0, 0, 0], (N, 1)).astype(np.int32)
    for i in range(N):
        t = rng.choice(V, 7, replace=False)
        x[i, :, t[0]], q[i, :, t[0]] = 0.0, 1.0
        x[i, :, t[1]], q[i, :, t[1]] = -rng.uniform(35.0, 37.0), 1e-10
        x[i, :, t[2:]] = -(60.0 + 240.0 * i / N) - rng.uniform(0.0, 2.0, (5, 1))
        tokens[i, 1:] = rng.choice(np.setdiff1d(np.arange(V), t), 4, replace=False)
    u = rng.random((N, T)).astype(np.float32)
    for dtype in (torch.float32, torch.bfloat16):
        got, ref = verify(L, torch.tensor(x, device="cuda").to(dtype), tokens, parent, u, 1.0, torch.tensor(q, device="cuda"))
        assert (ref[1] == 1).all()
        assert all(np.array_equal(g, r) for g, r in zip(got, ref)), int((got[2] != ref[2]).sum())
