"""Rows with a NaN or +inf have NaN for all of their numbers, whatever else they hold; the rows beside them are untouched by it."""
import numpy as np
import pytest

from oracle import vocab as O
from test_gpu_token_logprobs import check_forward, cuda, make, rows_of

pytestmark = pytest.mark.gpu


def spoilt(rows, vocab, seed):
    """Every row but each third is spoilt: one NaN, one +inf, NaN alone, NaN and -inf, +inf alone, NaN beside +inf."""
    x = make("plain", rows, vocab, seed)
    at = np.random.default_rng(seed).integers(0, vocab, rows)
    for r in range(rows):
        if r % 3 == 2:
            continue
        kind = r % 7
        if kind == 0:
            x[r, at[r]] = np.nan
        elif kind == 1:
            x[r, at[r]] = np.inf
        elif kind == 2:
            x[r] = np.nan
        elif kind == 3:
            x[r] = -np.inf
            x[r, at[r]] = np.nan
        elif kind == 4:
            x[r] = np.inf
        elif kind == 5:
            x[r, ::2] = np.nan
        else:
            x[r, at[r]] = np.nan
            x[r, (at[r] + 1) % vocab] = np.inf
    return x


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,vocab", [(20, 7), (20, 1999), (20, 20011), (520, 1999), (1, 30000)])
def test_rows_with_nan_and_infinity(rows, vocab, dtype):
    import paper_2506_06122_amd as R
    x, _ = rows_of(spoilt(rows, vocab, rows), dtype, 1)
    xs = x.float().cpu().numpy()
    t = np.random.default_rng(1).integers(-1, vocab, rows).astype(np.int32)
    top = min(5, vocab)
    got = R.rollout_token_logprobs(x, cuda(t), temperature=0.9, top=top)
    with np.errstate(invalid="ignore"):
        check_forward(xs, t, float(np.float32(0.9)), got, top)
        want = O.token_logprobs(xs, t, float(np.float32(0.9)), top)
    bad = np.isnan(want[1])
    assert bad.sum() >= rows // 2
    logp, entropy, stats, _, alt = (v.cpu().numpy() for v in got)
    assert np.array_equal(np.isnan(stats), np.isnan(want[2])) and np.isnan(stats[bad]).all()
    assert np.isnan(entropy[bad]).all() and np.isnan(alt[bad]).all()
    assert np.isnan(logp[bad & (t >= 0)]).all() and (logp[t < 0] == 0).all()


def test_lm_head_rows_with_nan_and_infinity():
    import torch
    import paper_2506_06122_amd as R
    rng = np.random.default_rng(4)
    for rows in (6, 200):
        h = rng.normal(0, 1, (rows, 64)).astype(np.float32)
        h[1, 5], h[3, 7], h[4] = np.nan, np.inf, np.nan   # (an infinity times weights of both signs: +inf somewhere)
        w = cuda(rng.normal(0, 1, (700, 64)).astype(np.float32)).to(torch.bfloat16)
        t = rng.integers(0, 700, rows).astype(np.int32)
        t[4] = -1
        logp, entropy, stats = (v.cpu().numpy() for v in R.rollout_head_logprobs(cuda(h).to(torch.bfloat16), w, cuda(t)))
        bad = np.isin(np.arange(rows), [1, 3, 4])
        for v in (entropy, stats[:, 0], stats[:, 1]):
            assert np.array_equal(np.isnan(v), bad)
        assert np.array_equal(np.isnan(logp), bad & (t >= 0)) and logp[4] == 0
