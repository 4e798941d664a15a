"""Log-probs straight from hidden states and the lm_head matrix, and both gradients, against oracle/vocab.py.

Tolerances (u = 2^-24).  A logit is a sum of K products of bf16 values, exact in fp32, added in fp32: off by K u of the sum
of their magnitudes at most (`fuzz`, per row the largest; the matrix instruction adds 32 at a time and may round each).  So
logp, entropy and stats are off by 2 fuzz beside the roundings of tests/test_gpu_token_logprobs.py.  The logits' gradient
is off by p (fuzz + those roundings) relative terms, and is rounded to bf16 once (2^-8, half a step) before the two products,
which add in fp32 and round once more to bf16."""
import numpy as np
import pytest

from oracle import vocab as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF = 2.0 ** -8


def inputs(rows, vocab, hidden, seed, pad=0, spread=2.5):
    import torch
    rng = np.random.default_rng(seed)

    def put(a):
        n, k = a.shape
        buf = torch.full((n, k + pad), 9.0, dtype=torch.bfloat16, device="cuda")
        buf[:, :k].copy_(torch.from_numpy(a.astype(np.float32)))
        return buf[:, :k]

    w = put(rng.normal(0, spread / np.sqrt(hidden), (vocab, hidden)))
    h = put(rng.normal(0, 1, (rows, hidden)))
    t = rng.integers(0, vocab, rows).astype(np.int32)
    t[0] = vocab - 1
    if rows > 2:
        t[1], t[2] = -1, vocab
    return h, w, t


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def cuda(a):
    import torch
    return None if a is None else torch.from_numpy(a).cuda()


def grads_of(rows, seed, entropy):
    rng = np.random.default_rng(seed + 2)
    g = rng.normal(0, 1, rows).astype(np.float32)
    h = rng.normal(0, 0.1, rows).astype(np.float32) if entropy else None
    skip = rng.random(rows) < 0.3
    g[skip] = 0
    if entropy:
        h[skip] = 0
    return g, h


def check(h, w, t, temperature, seed, entropy):
    import paper_2506_06122_amd as R
    hd, wd = host(h), host(w)
    rows, vocab = len(hd), len(wd)
    temperature = float(np.float32(temperature))
    fuzz = hd.shape[1] * U * (np.abs(hd) @ np.abs(wd).T).max(1) / temperature
    n = vocab / 256 + 60
    logp, ent, stats = O.head_logprobs(hd, wd, t, temperature)
    got = R.rollout_head_logprobs(h, w, cuda(t), temperature=temperature)
    gl, ge, gs = (host(v) for v in got)
    tol = 2 * fuzz + (n + 8) * U + 4 * U * (np.abs(logp) + 2 * np.abs(stats[:, 1]))
    assert np.all(np.abs(gl - logp) <= tol), (np.abs(gl - logp) / tol).max()
    tol_e = 4 * fuzz * (1 + np.log(vocab + 1)) + (3 * n + 40) * U * np.log(vocab + 2)
    assert np.all(np.abs(ge - ent) <= tol_e), (np.abs(ge - ent) / tol_e).max()
    assert np.all(np.abs(gs[:, 0] - stats[:, 0]) <= fuzz * temperature)
    assert np.all(np.abs(gs[:, 1] - stats[:, 1]) <= tol)

    g, e = grads_of(rows, seed, entropy)
    dh, dw = (host(v) for v in R.rollout_head_logprobs_grad(h, w, cuda(t), got[2], got[1], cuda(g), cuda(e), temperature=temperature))
    want_h, want_w, dx = O.head_logprobs_grad(hd, wd, t, temperature, g, e)
    x = hd @ wd.T
    lp = (x - stats[:, :1]) / temperature - stats[:, 1:]
    p, ee = np.exp(lp), np.zeros(rows) if e is None else np.abs(e)
    mag = (np.abs(lp) + stats[:, 1:] + 4)
    rel = 6 * U * mag + (n + 8) * U + 4 * fuzz[:, None]
    off = p * (np.abs(g)[:, None] + ee[:, None] * (mag + ent[:, None])) * rel + ee[:, None] * p * (mag * 6 * U + tol_e[:, None] + 4 * fuzz[:, None])
    off = (off + 8 * U * np.abs(g)[:, None]) / temperature
    off[(g == 0) & (ee == 0)] = 0
    off += BF * (np.abs(dx) + off)
    size = np.abs(dx) + off
    tol_h = off @ np.abs(wd) + (vocab + 32) * U * (size @ np.abs(wd))
    tol_w = off.T @ np.abs(hd) + (rows + 32) * U * (size.T @ np.abs(hd))
    assert np.all(np.abs(dh - want_h) <= tol_h + BF * (np.abs(want_h) + tol_h) + 2.0 ** -126), (np.abs(dh - want_h) - tol_h).max()
    assert np.all(np.abs(dw - want_w) <= tol_w + BF * (np.abs(want_w) + tol_w) + 2.0 ** -126), (np.abs(dw - want_w) - tol_w).max()
    # what a bound on every value lets through does not add up: the roundings are independent, so the errors' norms are a few steps
    for a, b in ((dh, want_h), (dw, want_w)):
        assert np.linalg.norm(a - b) <= 2 * BF * np.linalg.norm(b) + 1e-30
    return got, dh, dw


@pytest.mark.parametrize("rows,vocab,hidden", [(1, 1, 64), (1, 7, 64), (3, 300, 192), (16, 256, 128), (17, 257, 320), (33, 1000, 64),
                                               (64, 2049, 512), (65, 500, 64), (130, 1031, 256), (257, 4096, 128), (300, 50257, 64)])
@pytest.mark.parametrize("entropy", [False, True])
def test_sizes(rows, vocab, hidden, entropy):
    h, w, t = inputs(rows, vocab, hidden, rows, pad=8 * entropy)
    check(h, w, t, 0.7 if entropy else 1.0, rows, entropy)


def agree_with_the_logits_path(h, w, t):
    """Against float64 products on the GPU and the logits' own operator."""
    import paper_2506_06122_amd as R
    rows, hidden = h.shape
    g, e = map(cuda, grads_of(rows, 5, True))
    x = h.double() @ w.double().T
    got = R.rollout_head_logprobs(h, w, cuda(t))
    ref = R.rollout_token_logprobs(x.float(), cuda(t))
    fuzz = hidden * U * float((h.double().abs() @ w.double().abs().T).max())
    for a, b in zip(got, ref):
        assert float((a - b).abs().max()) <= 5 * fuzz + 200 * U * 20
    dh, dw = R.rollout_head_logprobs_grad(h, w, cuda(t), got[2], got[1], g, e)
    dx = R.rollout_token_logprobs_grad(x.float(), cuda(t), ref[2], ref[1], g, e).double()
    for a, b in ((dh, dx @ w.double()), (dw, dx.T @ h.double())):
        # two roundings to bf16, each at most 2^-8 relative to its value: their norms add up to less than 2^-7
        assert float((a.double() - b).norm() / b.norm()) <= 2 * BF


def test_tiles_of_every_size_agree_with_the_logits_path():
    """Large enough for the largest tiles."""
    for rows, vocab, hidden in ((1500, 12301, 192), (4096, 4099, 64), (513, 30001, 1536), (150, 50257, 128), (190, 50257, 64),
                                (310, 32001, 128), (430, 50257, 64), (128, 50257, 192), (65, 50257, 64), (420, 12301, 512)):
        agree_with_the_logits_path(*inputs(rows, vocab, hidden, 5))


def test_few_rows_of_an_lm_head_past_the_last_cache():
    h, w, t = inputs(128, 70001, 2048, 6)  # 287 MB
    for rows in (1, 9, 16, 20, 32, 50, 64, 100, 128):
        agree_with_the_logits_path(h[:rows], w, t[:rows])


def test_rows_without_gradient_and_no_rows():
    import torch
    import paper_2506_06122_amd as R
    h, w, t = inputs(70, 600, 64, 1)
    got = R.rollout_head_logprobs(h, w, cuda(t))
    zero = torch.zeros(70, device="cuda")
    dh, dw = R.rollout_head_logprobs_grad(h, w, cuda(t), got[2], got[1], zero, zero)
    assert not dh.any() and not dw.any()
    g = zero.clone()
    g[1:3] = 1.0        # rows without a target
    g[40] = -0.5
    dh, dw = R.rollout_head_logprobs_grad(h, w, cuda(t), got[2], got[1], g)
    one = torch.zeros(70, dtype=torch.bool, device="cuda")
    one[40] = True
    assert not dh[~one].any() and dh[40].any()
    lone = R.rollout_head_logprobs_grad(h[40:41], w, cuda(t[40:41].copy()), got[2][40:41].clone(), None, g[40:41].clone())
    assert torch.equal(lone[0][0], dh[40]) or float((lone[0][0] - dh[40]).abs().max()) <= 2 * BF * float(dh[40].abs().max())
    none = h[:0]
    logp, ent, stats = R.rollout_head_logprobs(none, w, zero[:0].int())
    assert len(logp) == 0
    dh, dw = R.rollout_head_logprobs_grad(none, w, zero[:0].int(), stats, ent, logp)
    assert dh.shape == (0, 64) and not dw.any()


def test_same_bits_on_another_stream_and_in_a_graph():
    import torch
    import paper_2506_06122_amd as R
    h, w, t = inputs(150, 3000, 128, 3)
    t, (g, e) = cuda(t), map(cuda, grads_of(150, 3, True))

    def both(h, stream=None):
        f = R.rollout_head_logprobs(h, w, t, temperature=1.2, stream=stream)
        return list(f) + list(R.rollout_head_logprobs_grad(h, w, t, f[2], f[1], g, e, temperature=1.2, stream=stream))

    want = both(h)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for a in (both(h), both(h, side.cuda_stream)):
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, want))
    held = h.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(held)
    for seed in range(3):
        y = inputs(150, 3000, 128, 30 + seed)[0]
        want = both(y)
        held.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))
