"""Pins of the windowed attention's oracle: masks against a pure-Python statement, values and gradients against torch in fp64."""
import numpy as np
import pytest
import torch

from oracle import window_oracle as wo


def test_masks_brute_force():
    rng = np.random.default_rng(1)
    for _ in range(60):
        Lq, Lk, chunk = (int(rng.integers(1, 12)) for _ in range(3))
        left, right, sinks = int(rng.integers(-1, 4)), int(rng.integers(-1, 3)), int(rng.integers(0, 3))
        n, start = int(rng.integers(0, Lk + 1)), int(rng.integers(-3, 12))
        M = wo.masks(1, Lq, Lk, left, right, sinks, chunk, start, [n])[0]
        for i in range(Lq):
            for j in range(Lk):
                p = start + i
                want = 0 <= p < n and j < n
                want = want and (right < 0 or j // chunk <= p // chunk + right)
                want = want and (left < 0 or j // chunk >= p // chunk - left or j // chunk < sinks)
                assert bool(M[i, j]) == want


def test_every_row_with_a_token_sees_its_own_position():
    M = wo.masks(2, 9, 9, 0, 0, 0, 1, 0, [9, 4])
    assert np.array_equal(M[0], np.eye(9, dtype=bool))
    assert np.array_equal(M[1], np.diag(np.arange(9) < 4))


@pytest.mark.parametrize("seed", range(4))
def test_values_and_gradients_against_torch(seed):
    rng = np.random.default_rng(seed)
    B, Hq, Hkv, L, d = 2, 4, 2, 13, 8
    Q, dO = rng.standard_normal((2, B, Hq, L, d))
    K, V = rng.standard_normal((2, B, Hkv, L, d))
    M = wo.masks(B, L, L, [3, -1, 0, 2][seed], [0, 0, 1, -1][seed], seed % 3, [1, 1, 4, 5][seed], 0, [L, 9])
    out, lse, mag = wo.window_attn(Q, K, V, M)
    (dq, dk, dv), _, _ = wo.window_attn_backward(Q, K, V, dO, M)
    q, k, v = (torch.tensor(x, requires_grad=True) for x in (Q, K, V))
    kk, vv = (x.repeat_interleave(2, 1) for x in (k, v))
    Mt = torch.tensor(M)[:, None]
    live = Mt.any(-1, keepdim=True)
    x = (q @ kk.transpose(2, 3) / d ** 0.5).masked_fill(~Mt, -1e300)
    o = torch.where(live, torch.softmax(x, -1) @ vv, 0.0)
    o.backward(torch.tensor(dO))
    for got, want in ((out, o), (dq, q.grad), (dk, k.grad), (dv, v.grad)):
        np.testing.assert_allclose(got, want.detach().numpy(), rtol=1e-10, atol=1e-12)
    want = torch.where(live.squeeze(-1), torch.logsumexp(x, -1), -torch.inf)
    np.testing.assert_allclose(lse, want.detach().numpy().reshape(lse.shape), rtol=1e-12)
    assert (mag >= np.abs(out) - 1e-12).all()
