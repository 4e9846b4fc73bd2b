"""The 64-bit reference of attention with a window against differences, and against the plain statement of its mask."""
import pytest
import torch

import attention_reference as ref


def operands(batch, heads, kv, N, M, d, seed):
    g = torch.Generator().manual_seed(seed)
    shape = lambda h, n: torch.randn((batch, h, n, d), dtype=torch.float64, generator=g)  # noqa: E731
    return shape(heads, N), shape(kv, M), shape(kv, M), shape(heads, N)


@pytest.mark.parametrize("N,M,window,sinks", [(5, 5, None, 0), (3, 7, 2, 1), (6, 4, None, 0), (4, 9, 3, 2), (1, 1, 1, 0)])
def test_mask_is_the_statement(N, M, window, sinks):
    seen = ref.visible(N, M, window, sinks)
    for i in range(N):
        p = i + M - N
        for j in range(M):
            assert bool(seen[i, j]) == (j <= p and (window is None or p - j < window or j < sinks))


@pytest.mark.parametrize("heads,kv,N,M,window,sinks", [(1, 1, 4, 4, None, 0), (4, 2, 5, 9, 3, 2), (3, 1, 6, 4, 2, 0), (2, 2, 3, 8, None, 0)])
def test_gradient_against_differences(heads, kv, N, M, window, sinks):
    """Central differences of the forward reference along random directions; the step leaves 1e-9 or so."""
    Q, K, V, dO = operands(2, heads, kv, N, M, 64, 5 + N)
    O, lse, _, _ = ref.forward(Q, K, V, window, sinks)
    grads, _ = ref.gradient(Q, K, V, O, lse, dO, window, sinks)
    h = 1e-4
    for which, grad in enumerate(grads):
        u = torch.randn(grad.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(which))
        value = []
        for sign in (1, -1):
            x = [Q, K, V]
            x[which] = x[which] + sign * h * u
            value.append((ref.forward(*x, window, sinks)[0] * dO).sum().item())
        want, got = (value[0] - value[1]) / (2 * h), (grad * u).sum().item()
        assert abs(got - want) <= 1e-6 * (1 + abs(want)), (which, got, want)
