"""Log-probs of given tokens from logits, entropies, alternatives and the logits' gradient, against oracle/vocab.py.

Tolerances (u = 2^-24, half a step of fp32 relative to the value).  A row's sum is made of at most n = vocab / 256 + 40
additions one after another, each off by u of the sum, of terms off by a few u each (the exponent's rounding is u |y| with
the term 2^y: |y| 2^y < 0.54), so ln S is off by (n + 8) u.  logp adds the roundings of its terms; entropy = ln S + a sum
of the same kind, at most n + 16 roundings of a value no larger than ln vocab each.  A gradient's exponent y - ln S /ln 2
is rounded a few times relative to its terms, then the result once to its type, by half a step."""
import numpy as np
import pytest

from oracle import vocab as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = ["float32", "bfloat16", "float16"]


def torch_type(name):
    import torch
    return getattr(torch, name)


def rows_of(values, dtype, pad=0, shift=0):
    """`values` on the GPU, `pad` spare values behind every row, the first row `shift` values past an aligned address;
    returns the view and the buffer around it."""
    import torch
    rows, vocab = values.shape
    buf = torch.full((shift + rows * (vocab + pad),), 77.0, dtype=torch_type(dtype), device="cuda")
    view = buf[shift:].as_strided((rows, vocab), (vocab + pad, 1))
    view.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    return view, buf


def make(kind, rows, vocab, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 2.5, (rows, vocab)).astype(np.float32)
    if kind == "ties":
        x = rng.integers(-2, 3, (rows, vocab)).astype(np.float32)
    elif kind == "constant":
        x[:] = -1.5
    elif kind == "banned":     # about one id in ten is left, in the last row two
        x[rng.random((rows, vocab)) < 0.9] = -np.inf
        x[:, vocab // 2] = 0.25
        x[-1] = -np.inf
        x[-1, [0, vocab - 1]] = 1.0, 2.0
    elif kind == "empty":      # rows of nothing, among them the first
        x[::2] = -np.inf
    elif kind == "lowest":     # a mask of the type's lowest value, over all of some rows
        x[:, ::3] = -65504.0
        x[0] = -65504.0
    elif kind == "huge":       # differences that do not fit fp32's range of exponents, or of values
        x *= 3e3
        x[0, 0] = 6e4
    elif kind == "spike":
        x[:, vocab - 1] += 40.0
    elif kind == "descending":
        x = np.sort(x, 1)[:, ::-1].copy()
    return x


def targets_of(rows, vocab, seed):
    t = np.random.default_rng(seed + 1).integers(0, vocab, rows).astype(np.int32)
    t[0] = vocab - 1
    if rows > 2:
        t[1], t[2] = -1, vocab
    return t


def check_forward(x, t, temperature, got, top):
    logp, entropy, stats, ids, alt = O.token_logprobs(x, t, temperature, top)
    # a log-prob below fp32's range is -inf in fp32: two values of the full range, 6.8e38 apart, over T = 1/4
    logp, alt = (np.where(v < -2.0 ** 128, -np.inf, v) for v in (logp, alt))
    n = x.shape[1] / 256 + 40
    log_s = np.where(np.isfinite(stats[:, 1]), stats[:, 1], 0.0)
    tol_s = (n + 8) * U
    g = [None if v is None else v.cpu().numpy().astype(np.float64) for v in got]
    assert np.array_equal(np.isfinite(g[0]), np.isfinite(logp)) and np.array_equal(np.isnan(g[0]), np.isnan(logp))
    held = np.isfinite(logp)
    off = np.abs(g[0] - logp)[held]
    assert np.all(off <= tol_s + 4 * U * (np.abs(logp) + 2 * np.abs(log_s))[held]), off.max()
    assert np.array_equal(g[0][~held & ~np.isnan(logp)], logp[~held & ~np.isnan(logp)])
    held = np.isfinite(entropy)
    assert np.array_equal(held, np.isfinite(g[1]))
    assert np.all(np.abs(g[1] - entropy)[held] <= tol_s + (2 * n + 32) * U * np.log(max(x.shape[1], 2))), np.abs(g[1] - entropy).max()
    clean = ~np.isnan(stats[:, 1])
    assert np.array_equal(g[2][clean, 0], stats[clean, 0])
    assert np.array_equal(np.isnan(g[2][:, 1]), ~clean)
    fin = np.isfinite(stats[:, 1])
    assert np.all(np.abs(g[2][fin, 1] - stats[fin, 1]) <= tol_s + U * np.abs(log_s[fin]))
    assert np.array_equal(g[2][~fin & clean, 1], stats[~fin & clean, 1])
    if top:
        assert np.array_equal(g[3], ids)
        held = np.isfinite(alt)
        assert np.array_equal(g[4][~held & ~np.isnan(alt)], alt[~held & ~np.isnan(alt)])
        lim = tol_s + 4 * U * (np.abs(np.where(held, alt, 0)) + 2 * np.abs(log_s)[:, None])
        assert np.all(np.abs(g[4] - alt)[held] <= lim[held])
        assert np.array_equal(np.isnan(g[4]), np.isnan(alt))


def half_step(dtype, v):
    """Half a step of a type at values v, its smallest step included."""
    eps, least = {"float32": (2.0 ** -24, 2.0 ** -150), "bfloat16": (2.0 ** -8, 2.0 ** -134), "float16": (2.0 ** -11, 2.0 ** -25)}[dtype]
    return eps * np.abs(v) + least


def check_grad(x, t, temperature, g, h, got, dtype, log_s, slack=0.0):
    want = O.token_logprobs_grad(x, t, temperature, g, h)
    _, entropy, stats, _, _ = O.token_logprobs(x, None, temperature)
    ls = np.where(np.isfinite(log_s), log_s, 0.0)[:, None]
    with np.errstate(invalid="ignore"):
        lp = np.where(np.isfinite(x), (x - stats[:, :1]) / temperature - ls, -np.inf)
    p = np.exp(np.where(np.isnan(lp), -np.inf, lp))
    mag = np.where(p > 0, np.abs(lp), 0.0) + ls + 4          # the exponent's terms, in nats
    hh = np.zeros(len(x)) if h is None else np.abs(h)
    ent = np.nan_to_num(entropy)
    n = x.shape[1] / 256 + 40
    # p off by 6 u of its exponent's terms and by the forward pass' ln S; the entropy's part by the entropy's error too
    tol = p * (np.abs(g)[:, None] + hh[:, None] * (mag + ent[:, None])) * (6 * U * mag + (n + 8) * U)
    tol += hh[:, None] * p * (mag * 6 * U + (3 * n + 40) * U * np.log(max(x.shape[1], 2)))
    tol = (tol + 8 * U * np.abs(g)[:, None]) / temperature + slack
    got = got.float().cpu().numpy().astype(np.float64)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    off = np.abs(got - want) - tol - half_step(dtype, np.abs(want) + tol) * 1.001
    assert np.all(off[~nan] <= 2.0 ** -126), (off[~nan].max(), np.unravel_index(np.nanargmax(off), off.shape))


def grads_of(rows, seed, entropy):
    rng = np.random.default_rng(seed + 2)
    g = rng.normal(0, 1, rows).astype(np.float32)
    g[rows // 2] = 0.0
    h = rng.normal(0, 0.1, rows).astype(np.float32) if entropy else None
    if entropy:
        h[rows // 2] = 0.0
    return g, h


def cuda(a):
    import torch
    return None if a is None else torch.from_numpy(a).cuda()


SIZES = [(1, 1), (2, 2), (3, 7), (5, 33), (4, 255), (3, 257), (2, 2047), (1, 4097), (7, 32001), (1, 151936), (1030, 515), (40, 9001)]


@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_sizes_strides_and_alignments(rows, vocab, dtype):
    import paper_2506_06122_amd as R
    for i, (pad, shift, top, temperature) in enumerate([(0, 0, 1, 1.0), (1, 3, 20, 0.7), (8, 0, 64, 1.3), (5, 1, 0, 1.0)]):
        top = min(top, vocab)
        x, _ = rows_of(make("plain", rows, vocab, i), dtype, pad, shift)
        t = targets_of(rows, vocab, i)
        got = R.rollout_token_logprobs(x, cuda(t), temperature=temperature, top=top)
        xs = x.float().cpu().numpy()
        check_forward(xs, t, np.float32(temperature), got, top)
        g, h = grads_of(rows, i, i % 2 == 1)
        out, buf = rows_of(np.zeros((rows, vocab), np.float32), dtype, 3 - i % 2, i)
        out.fill_(5.0)
        R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h), temperature=temperature, out=out)
        check_grad(xs, t, np.float32(temperature), g, h, out, dtype, got[2][:, 1].cpu().numpy().astype(np.float64))
        gaps = buf.float().cpu().numpy()
        inside = np.zeros(len(gaps), bool)
        for r in range(rows):
            inside[i + r * (vocab + 3 - i % 2):][:vocab] = True
        assert (gaps[~inside] == 77.0).all(), "a value between the rows was written"


@pytest.mark.parametrize("kind", ["ties", "constant", "banned", "empty", "lowest", "huge", "spike", "descending"])
@pytest.mark.parametrize("rows,vocab", [(3, 37), (6, 5003), (2, 50257), (1027, 1500)])
def test_rows_that_are_hard(kind, rows, vocab):
    import paper_2506_06122_amd as R
    for dtype, top in (("float32", 20), ("bfloat16", 37)):
        x, _ = rows_of(make(kind, rows, vocab, 7), dtype, 1)
        t = targets_of(rows, vocab, 7)
        xs = x.float().cpu().numpy()
        got = R.rollout_token_logprobs(x, cuda(t), temperature=0.9, top=top)
        check_forward(xs, t, np.float32(0.9), got, top)
        g, h = grads_of(rows, 7, True)
        out = R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h), temperature=0.9)
        check_grad(xs, t, np.float32(0.9), g, h, out, dtype, got[2][:, 1].cpu().numpy().astype(np.float64))


def test_the_lowest_fp32_value_everywhere_is_a_uniform_row():
    import paper_2506_06122_amd as R
    x = np.full((2, 3001), np.finfo(np.float32).min, np.float32)
    x[1, 7] = np.finfo(np.float32).max
    got = R.rollout_token_logprobs(cuda(x), cuda(np.array([5, 7], np.int32)), temperature=0.25, top=3)
    check_forward(x, np.array([5, 7]), 0.25, got, 3)


def test_nan_and_infinite_rows():
    import paper_2506_06122_amd as R
    for vocab in (40, 6000, 50257):
        x = make("plain", 6, vocab, 1)
        x[1, vocab // 3] = np.nan
        x[2, vocab - 1] = np.inf
        x[3] = np.nan
        x[4, ::2] = np.nan
        t = np.array([1, 2, 3, 4, 5, -1], np.int32)
        got = R.rollout_token_logprobs(cuda(x), cuda(t), top=30)
        check_forward(x, t, 1.0, got, 30)
        g = np.array([1, 1, 1, 1, 0, 1], np.float32)
        out = R.rollout_token_logprobs_grad(cuda(x), cuda(t), got[2], got[1], cuda(g))
        check_grad(x, t, 1.0, g, None, out, "float32", got[2][:, 1].cpu().numpy().astype(np.float64))


def test_no_targets_and_no_rows():
    import torch
    import paper_2506_06122_amd as R
    x = make("plain", 3, 700, 2)
    got = R.rollout_token_logprobs(cuda(x), None, top=2)
    assert got[0].tolist() == [0.0, 0.0, 0.0]
    check_forward(x, None, 1.0, got, 2)
    g, h = grads_of(3, 1, True)
    out = R.rollout_token_logprobs_grad(cuda(x), None, got[2], got[1], cuda(g), cuda(h))
    check_grad(x, None, 1.0, g, h, out, "float32", got[2][:, 1].cpu().numpy().astype(np.float64))
    none = torch.zeros(0, 700, device="cuda")
    logp, entropy, stats, ids, alt = R.rollout_token_logprobs(none, torch.zeros(0, dtype=torch.int32, device="cuda"), top=2)
    assert len(logp) == 0 and stats.shape == (0, 2) and ids.shape == alt.shape == (0, 2)
    assert R.rollout_token_logprobs_grad(none, None, stats, entropy, logp).shape == (0, 700)


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(dtype):
    import paper_2506_06122_amd as R
    x, buf = rows_of(make("plain", 5, 3333, 4), dtype, 7, 1)
    t = targets_of(5, 3333, 4)
    got = R.rollout_token_logprobs(x, cuda(t))
    g, h = grads_of(5, 4, True)
    want = R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h))
    same = R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h), out=x)
    assert same.data_ptr() == x.data_ptr() and (x == want).all()
    assert (buf[1 + 3333:1 + 3340] == 77.0).all()


def test_gradients_beside_their_logits():
    import torch
    import paper_2506_06122_amd as R
    wide = torch.full((6, 2 * 1001 + 3), 7.0, device="cuda")
    x, out = wide[:, :1001], wide[:, 1003:2004]
    x.copy_(torch.from_numpy(make("plain", 6, 1001, 8)))
    t = targets_of(6, 1001, 8)
    got = R.rollout_token_logprobs(x, cuda(t))
    g, h = grads_of(6, 8, True)
    want = R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h))
    held = x.clone()
    R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h), out=out)
    assert torch.equal(out, want) and torch.equal(x, held)
    assert (wide[:, 1001:1003] == 7.0).all() and (wide[:, 2004:] == 7.0).all()
    with pytest.raises(R.RolloutError):
        R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), cuda(h), out=wide[:, 1000:2001])


def test_rows_past_32_bits():
    import torch
    import paper_2506_06122_amd as R
    vocab, stride = 1003, (1 << 31) + 9
    buf = torch.zeros(stride + vocab + 1, dtype=torch.bfloat16, device="cuda")
    x = buf[1:].as_strided((2, vocab), (stride, 1))
    x.copy_(torch.from_numpy(make("plain", 2, vocab, 9)))
    t = np.array([3, 900], np.int32)
    xs = x.float().cpu().numpy()
    got = R.rollout_token_logprobs(x, cuda(t), top=5)
    check_forward(xs, t, 1.0, got, 5)
    g = np.array([1.0, -2.0], np.float32)
    out = R.rollout_token_logprobs_grad(x, cuda(t), got[2], got[1], cuda(g), out=x)
    check_grad(xs, t, 1.0, g, None, out, "bfloat16", got[2][:, 1].cpu().numpy().astype(np.float64))


def test_same_bits_again_on_another_stream_and_in_a_graph():
    import torch
    import paper_2506_06122_amd as R
    x = cuda(make("banned", 5, 20011, 6))
    t, (g, h) = cuda(targets_of(5, 20011, 6)), map(cuda, grads_of(5, 6, True))

    def both(x, stream=None):
        f = R.rollout_token_logprobs(x, t, temperature=0.8, top=9, stream=stream)
        return list(f) + [R.rollout_token_logprobs_grad(x, t, f[2], f[1], g, h, temperature=0.8, stream=stream)]

    want = both(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for a in (both(x), both(x, side.cuda_stream)):
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, want))
    held = x.clone()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(held)
    with torch.cuda.graph(other):
        out2 = both(x)
    for seed in range(3):
        y = cuda(make("plain", 5, 20011, 20 + seed))
        want_y = both(y)
        held.copy_(y)
        with torch.cuda.stream(side):   # two graphs at a time: each has its own workspace
            other.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want_y))
        assert all(torch.equal(p, q) for p, q in zip(out2, want))
        del y, want_y
        torch.cuda.synchronize()


def test_gradient_against_differences_of_the_forward_pass():
    import paper_2506_06122_amd as R
    rng = np.random.default_rng(11)
    x = rng.normal(0, 2, (4, 301)).astype(np.float32)
    t, g, h = np.array([3, 300, -1, 40], np.int32), rng.normal(size=4).astype(np.float32), rng.normal(size=4).astype(np.float32)
    got = R.rollout_token_logprobs(cuda(x), cuda(t), temperature=1.1)
    dx = R.rollout_token_logprobs_grad(cuda(x), cuda(t), got[2], got[1], cuda(g), cuda(h), temperature=1.1).cpu().numpy()
    for k in range(5):
        way = rng.normal(size=x.shape)

        def f(s):
            logp, entropy, *_ = O.token_logprobs(x + s * way, t, np.float32(1.1))
            return float(g @ logp + h @ entropy)

        slope = (f(1e-5) - f(-1e-5)) / 2e-5
        # 64-bit differences are good to 1e-9; the gradient's 1204 values to about 20 u of their row's weight
        assert abs(slope - float(np.sum(dx * way))) <= 1e-6 * (np.abs(dx) * np.abs(way)).sum() + 1e-8
