"""Rows with one nearly certain token, as a trained model's are: the statistics are taken relative to the row's largest logit.

Tolerances.  The largest logit's term is 1 exactly; the sum s = 1 + d that a thread, a warp, a team and a cluster add up rounds
at most 16 times within the batch of that logit, once per batch (9 of them here), and 13 times on the way to the row's sum: 38
roundings of 2^-24 at worst, 2.3e-6 in all, and if they are independent and evenly spread a root mean square of
2^-24 sqrt(38 / 3) = 2.1e-7.  A term below the largest is off by 2^-17 of itself at worst (two roundings of an exponent up to 64
and the exponential), which enters as 2^-17 d in ln s and 2^-17 d |ln p| <= 2^-17 45 d in the entropy.  A value itself is rounded
to 2^-24 of it."""
import numpy as np
import pytest
import torch

import paper_2608_12573_b200 as profk
from oracle import decode as oracle
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,k", [(3, 0), (3, 5), (311, 0), (311, 5), (311, 40)])
def test_rows_with_one_nearly_certain_token(dtype, rows, k):
    vocab = 50001
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + k)
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    x.scatter_(1, tokens[:, None], torch.linspace(18, 34, rows, device="cuda")[:, None] + torch.rand(rows, 1, generator=g, device="cuda"))
    x = x.to(DTYPES[dtype])
    r = profk.logprobs(x, tokens, k=k)
    host = x.double().cpu().numpy()
    want = [oracle.logprobs_row(host[i], int(tokens[i])) for i in range(rows)]
    lp, ent = (np.array([w[key] for w in want]) for key in ("logprob", "entropy"))
    got_lp, got_ent = (t.double().cpu().numpy() for t in (r.logprob, r.entropy))
    assert (got_lp <= 0).all() and (got_ent >= 0).all()
    d = -np.expm1(lp)                                                # the other tokens' probability
    for got, exact, spread in ((got_lp, lp, 1), (got_ent, ent, 45)):
        rounded = 2.0 ** -17 * spread * d + 2.0 ** -24 * np.abs(exact)
        off = np.abs(got - exact)
        assert (off <= 2.3e-6 + rounded).all(), off.max()
        if rows > 100:
            certain = d < 2.0 ** -12
            assert certain.sum() > 100
            rms = np.sqrt(np.mean(off[certain] ** 2))
            assert rms <= 2.1e-7 + np.sqrt(np.mean(rounded[certain] ** 2)), rms
    if k:
        assert (r.top_logprobs <= 0).all() and torch.equal(r.top_tokens[:, 0], tokens) and torch.equal(r.top_logprobs[:, 0], r.logprob)
