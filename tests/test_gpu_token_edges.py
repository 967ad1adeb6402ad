"""The ends of the token operators' ranges: the largest sums, scores and values, results on other streams, and the launch forms that few calls reach."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import pick
from tests.test_gpu_token_cache import BF, HF, Case, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dc():
    import paper_2609_35115_b200 as dc
    dc.load_library()
    return dc


# ---- sampling ------------------------------------------------------------------------------------------------------------------


def test_masses_of_flat_rows_of_the_largest_vocabulary(dc):
    """Rows that begin off a 16-byte border: a thread adds up to 260 weights close to one, whose sum passes 2^53 units of 2^-45.  The last tokens weigh nothing, so
    that the last kept one lies at the end of the part of a warp whose threads have that many."""
    n, vocab, kept = 150, 262144, 262144 - 6276
    rng = np.random.default_rng(21)
    g = torch.Generator(device="cuda").manual_seed(21)
    l = torch.randn(n, vocab + 1, generator=g, device="cuda")[:, :vocab]
    l[:, kept:] = -torch.inf
    u = torch.tensor(np.where(np.arange(n) % 3 == 0, rng.random(n), 1.0), dtype=torch.float32, device="cuda")
    T = torch.full((n,), 1e3, device="cuda")
    tokens, probs = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), 9.0, device="cuda")
    dc.sample_tokens(l, u, temperature=T, tokens=tokens, probs=probs)
    got, share = tokens.tolist(), probs.tolist()
    for r in range(n):
        if r % 3:      # u = 1: the last kept token, whatever the others weigh
            assert got[r] == kept - 1 and 0 < share[r] < 1e-5, r
        else:
            want, p = pick(l[r].double().cpu().numpy(), float(u[r]), 1e3)
            assert got[r] == want and abs(share[r] - p) <= 2.0 ** -24 * p * 1.001, r
