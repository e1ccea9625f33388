"""Products over a very long K: what the tensor cores cut from a running sum stays bounded, whatever the number of rows."""
import pytest
import torch

from tests.dense_util import E4M3, ctx, gen, status

pytestmark = pytest.mark.gpu
F32, F16 = torch.float32, torch.float16
K = 1 << 20


@pytest.mark.parametrize("ab", [F16, E4M3])
def test_sums_of_one_sign(ab):
    """Every term positive, the worst case: each of a chain's instructions (32 bytes of K) may cut one step, 2^-23, of the running sum.
    A chain is at most 64 k-blocks of 4 instructions in one accumulator (fp32 out), 256 (16 bits out); what the chains give is added
    with roundings, 2^-24 each, in at most K bytes / 1280 additions.  Then the output's half step."""
    g = gen(7)
    n, rows, es = 64, 300, 2 if ab == F16 else 1
    a, w = (torch.rand(r, K, generator=g, device="cuda").mul_(0.25).add_(0.01).to(ab) for r in (rows, n))
    want = torch.zeros(rows, n, device="cuda", dtype=torch.float64)
    for i in range(0, K, 1 << 17):
        want += a[:, i:i + (1 << 17)].double() @ w[:, i:i + (1 << 17)].double().T
    additions = K * es / 1280 * 2.0 ** -24
    for m in (1, 4, 40, 70, 140, 300):
        for c_t, chain, half in ((F32, 256 * 2.0 ** -23, 2.0 ** -24), (F16, 1024 * 2.0 ** -23, 2.0 ** -11)):
            out = torch.empty(m, n, device="cuda", dtype=c_t)
            ctx().linear(a[:m], w, out)
            bound = chain + additions + half
            assert float(((out.double() - want[:m]) / want[:m]).abs().max()) <= bound, (m, c_t)
    assert status() == 0
