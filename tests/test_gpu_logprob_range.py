"""Log-probs and gradients over the whole range of logits and temperatures that the calls accept: masks of large finite values over
blocks of a row, over whole threads, parts and rows; temperatures down to 1e-10.  Tolerances as in test_gpu_token_logprobs.py."""
import numpy as np
import pytest

from oracle import vocab as O
from test_gpu_token_logprobs import check_forward, check_grad, cuda, rows_of

pytestmark = pytest.mark.gpu
BF = 2.0 ** -8

FILLS = [-65504.0, -1e9, -1e10, -1e12, -1e20, -1e30, -1e38, -np.inf]


def masked(vocab, fills, seed):
    """Five rows of each fill: everywhere, the first and the last nine tenths, all but one, every third value."""
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 2.5, (5 * len(fills), vocab)).astype(np.float32)
    for i, fill in enumerate(fills):
        all_, first, last, but_one, third = x[5 * i:5 * i + 5]
        all_[:] = fill
        first[:vocab * 9 // 10] = fill
        last[vocab // 10:] = fill
        kept = but_one[vocab // 2]
        but_one[:] = fill
        but_one[vocab // 2] = kept
        third[::3] = fill
    return x


def check(x, dtype, temperature, top, seed):
    import paper_2506_06122_amd as R
    rng = np.random.default_rng(seed)
    t32 = float(np.float32(temperature))
    x, _ = rows_of(x, dtype, 1)
    rows, vocab = x.shape
    t = np.where(rng.random(rows) < 0.5, rng.integers(0, vocab, rows), x.float().argmax(1).cpu().numpy()).astype(np.int32)
    xs = x.float().cpu().numpy()
    got = R.rollout_token_logprobs(x, cuda(t), temperature=temperature, top=top)
    with np.errstate(invalid="ignore"):
        check_forward(xs, t, t32, got, top)
        g = rng.normal(0, 1, rows).astype(np.float32)
        for h in (None, rng.normal(0, 0.1, rows).astype(np.float32)):
            out = R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h), temperature=temperature)
            check_grad(xs, t, t32, g, h, out, dtype, got[2][:, 1].cpu().numpy().astype(np.float64))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("temperature", [0.25, 0.6, 0.7, 1.0, 1.3, 2.0, 1e3])
@pytest.mark.parametrize("vocab,times", [(1999, 1), (50257, 1), (2309, 15)])  # one part; many; a workgroup to a row of several chunks
def test_blocks_of_a_finite_mask(vocab, times, temperature, dtype):
    x = masked(vocab, FILLS, vocab)
    check(np.tile(x, (times, 1)), dtype, temperature, 7, 1)


@pytest.mark.parametrize("temperature", [1.5, 2.0, 3.0])
def test_rows_of_the_lowest_value(temperature):
    for dtype in ("float32", "bfloat16", "float16"):
        import torch
        x = np.full((3, 5003), float(torch.finfo(getattr(torch, dtype)).min), np.float32)
        x[1, 4000:] = 0.5
        check(x, dtype, temperature, 3, 2)


# (float16 does not hold gradients of more than 65504)
@pytest.mark.parametrize("temperature,dtype", [(1e-3, "float16")] + [(t, d) for t in (1e-3, 1e-5, 1e-6, 1e-7, 1e-8) for d in ("float32", "bfloat16")])
@pytest.mark.parametrize("size", [2.5, 1e3, 1.5e4])
def test_small_temperatures(size, temperature, dtype):
    rng = np.random.default_rng(int(size))
    x = rng.normal(0, 1, (40, 9001)).astype(np.float32)
    x = np.clip(x, -4, 4) * np.float32(size)
    x[::4, 100:4000] = -np.inf
    check(x, dtype, temperature, 5, 3)


@pytest.mark.parametrize("exponent", [20, 21, 22, 23, 24, 30, 31, 33])
def test_neighbouring_values_of_large_exponents(exponent):
    """Exponents x log2(e) / T on both sides of 2^k, neighbouring fp32 values: differences of a few units up to some hundreds."""
    for sign in (1.0, -1.0):
        for temperature in (1.0, 0.7, 1e-6):
            at = sign * 2.0 ** exponent * temperature / 1.4426950408889634
            steps = np.random.default_rng(exponent).integers(-60, 61, (6, 20011))
            x = (at * (1 + steps * 2.0 ** -23)).astype(np.float32)
            x[1::2, :15000] = np.float32(at * (1 - sign * 2.0 ** -10))   # whole parts on one side
            check(x, "float32", temperature, 4, 4)


@pytest.mark.parametrize("temperature", [1e-3, 1e-6, 1e-7, 1e-8])
@pytest.mark.parametrize("rows,vocab", [(5, 1000), (130, 3001), (300, 50257)])
def test_lm_head_of_whole_numbers(rows, vocab, temperature):
    """Logits that are whole numbers come out exact, whatever the temperature makes of them."""
    import torch
    import paper_2506_06122_amd as R
    rng = np.random.default_rng(rows)
    h, w = rng.integers(-2, 3, (rows, 64)).astype(np.float64), rng.integers(-3, 4, (vocab, 64)).astype(np.float64)
    t32 = float(np.float32(temperature))
    hd, wd = (cuda(a.astype(np.float32)).to(torch.bfloat16) for a in (h, w))
    x = h @ w.T
    t = np.where(rng.random(rows) < 0.5, rng.integers(0, vocab, rows), x.argmax(1)).astype(np.int32)
    got = R.rollout_head_logprobs(hd, wd, cuda(t), temperature=temperature)
    check_forward(x, t, t32, list(got) + [None, None], 0)
    g, e = rng.normal(0, 1, rows).astype(np.float32), rng.normal(0, 0.1, rows).astype(np.float32)
    dh, dw = R.rollout_head_logprobs_grad(hd, wd, cuda(t), got[2], got[1], cuda(g), cuda(e), temperature=temperature)
    want_h, want_w, _ = O.head_logprobs_grad(h, w, t, t32, g, e)
    for a, b in ((dh, want_h), (dw, want_w)):
        # two roundings to bf16, each at most 2^-8 relative to its value: their norms add up to less than 2^-7
        assert np.linalg.norm(a.double().cpu().numpy() - b) <= 2 * BF * np.linalg.norm(b)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("temperature", [1e-9, 1e-10, 1e-20, 1e-37])
def test_gradients_at_the_smallest_temperatures(temperature, dtype):
    """The entropy's part of a masked value's gradient is 0, however large 1 / T."""
    x = masked(5003, [-65504.0, -1e30, -np.inf], 11)
    x[::2, 100:200] = x.max(1)[::2, None]  # ties: a distribution over some
    check(x, dtype, temperature, 3, 5)


@pytest.mark.parametrize("temperature", [1e-10, 1e-30])
def test_lm_head_gradients_at_the_smallest_temperatures(temperature):
    for rows, vocab in ((5, 1000), (130, 3001)):
        test_lm_head_of_whole_numbers(rows, vocab, temperature)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("temperature", [1e9, 1e30, 3e38])
def test_large_temperatures(temperature, dtype):
    """Banned ids stay banned where log2(e) / T is below fp32's normal range."""
    x = masked(5003, [-65504.0, -1e30, -3e38, -np.inf], 12)
    x[:, 7] = 3e38 if dtype == "float32" else 2.5
    check(x, dtype, temperature, 3, 6)
