"""The loss against a teacher and its gradient at temperatures near both ends of the range of fp32, against the definition in 64 bits."""
import numpy as np
import pytest

from paper_2605_24058_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    return torch


@pytest.mark.parametrize("k", [1, 5, 80])
@pytest.mark.parametrize("V", [100, 5003, 40000])
@pytest.mark.parametrize("u", [1.2e-38, 1e-36, 1e-30, 1e-12, 1e-3, 0.1, 1.0, 30.0, 1e6, 1e12, 1e18])
def test_small_and_large_temperatures(torch, u, V, k):
    rng, T = np.random.default_rng(V + k), 7
    u = float(np.float32(u))
    z = (rng.standard_normal((T, V)) * 30).astype(np.float32)
    index = np.stack([rng.choice(V, size=k, replace=False) for _ in range(T)]).astype(np.int32)
    top = (rng.standard_normal((T, k)) * 20).astype(np.float32)
    index[0, 0] = z[0].argmax()
    top[0, 0] = 200              # a teacher who agrees
    cu = lambda a: torch.from_numpy(a).cuda()
    ones = torch.ones(T, device="cuda")
    loss, grad = binding.lordba_distill(cu(z), cu(index), cu(top), temperature=u, d_loss=ones)
    loss2, kept = binding.lordba_distill(cu(z), cu(index), cu(top), temperature=u)
    grad2 = binding.lordba_distill_backward(ones, cu(z), kept, cu(index), cu(top), temperature=u)
    zd, td, i = torch.from_numpy(z).double(), torch.from_numpy(top).double(), torch.from_numpy(index).long()
    lse = lambda v: u * torch.logsumexp((v - v.amax(1, keepdim=True)) / u, 1, keepdim=True) + v.amax(1, keepdim=True)     # u times it
    log_p, log_q = td - lse(td), zd - lse(zd)                                                                             # u times each
    p, q = (log_p / u).exp(), (log_q / u).exp()
    pieces = p * (log_p - log_q.gather(1, i))
    want = u * pieces.sum(1)
    # a probability: 4 roundings of an argument up to A (beyond 104 it is 0), the exponential's 2^-22, the sums of V and k entries.  The difference of the logarithms, times u: 4 roundings of
    # the logits' span and of u times logarithms up to log V
    span, A = 300.0, min(104.0, 300.0 / u) + np.log(V)
    rel = 2 * (4 * 2.0 ** -24 * A + 2.0 ** -22 + (V / 64 + 64) * 2.0 ** -24)
    err = u * (pieces.abs().sum(1) * (rel + k * 2.0 ** -24) + 4 * 2.0 ** -24 * (span + 2 * u * (np.log(V) + 1)) + u * rel) + 2.0 ** -148
    for got in (loss, loss2):
        got = got.double().cpu()
        assert bool((abs(got - want) <= 1.01 * err).all()), (got, want, err)
    p = torch.zeros_like(q).scatter_add_(1, i, p)
    want, err = u * (q - p), u * (q + p) * (rel + 2.0 ** -21) + 2.0 ** -148 + u * 2.0 ** -100
    for got in (grad, grad2):
        got = got.double().cpu()
        assert bool((abs(got - want) <= 1.01 * err).all()), float((abs(got - want) / err).max())
