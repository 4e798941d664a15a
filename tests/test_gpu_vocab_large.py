"""The operators at the vocabulary's ends where launches have more than 2^32 threads or rows are the longest that there are.
Tens of GB each, made on the GPU."""
import pytest

U, BF = 2.0 ** -24, 2.0 ** -8

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    import torch
    if torch.cuda.get_device_properties(0).total_memory < 120 << 30:
        pytest.skip("needs 120 GB of GPU memory")
    yield
    torch.cuda.empty_cache()


def test_the_most_rows_of_logits():
    import torch
    import paper_2506_06122_amd as R
    torch.manual_seed(1)
    rows = (1 << 24) - 64
    x = torch.randn(rows, 5, device="cuda").bfloat16()
    t = torch.randint(0, 5, (rows,), device="cuda", dtype=torch.int32)
    g = torch.randn(rows, device="cuda")
    logp, ent, stats, ids, _ = R.rollout_token_logprobs(x, t, top=1)
    lp = torch.log_softmax(x.double(), 1)
    # |x - max| < 13: ln S is off by its exponents' (2 x 18 + 8) U, the difference by 2 x 13 U, the logarithm by a few
    assert float((logp - lp.gather(1, t.long()[:, None])[:, 0]).abs().max()) <= 80 * U
    assert bool((x.gather(1, ids.long()) == x.max(1, keepdim=True).values).all())
    got = R.rollout_token_logprobs_grad(x, t, stats, ent, g)
    want = -lp.exp() * g[:, None]
    want.scatter_add_(1, t.long()[:, None], g[:, None].double())
    off = (got - want).abs() - BF * want.abs() - 100 * U * g.abs()[:, None]
    assert float(off.max()) <= 0


def test_many_odd_rows_of_an_embedding():
    import torch
    import paper_2506_06122_amd as R
    torch.manual_seed(2)
    n, hidden = (1 << 20) + 3, 4100  # a value to a thread: past 2^32 threads
    table = torch.randn(11, hidden, device="cuda").bfloat16()
    tokens = torch.randint(-1, 11, (n,), device="cuda", dtype=torch.int32)
    out = R.rollout_embed(table, tokens)
    rows = torch.cat([table, torch.zeros(1, hidden, device="cuda").bfloat16()])  # -1: the last
    for i in range(0, n, 1 << 17):
        assert torch.equal(out[i:i + (1 << 17)], rows[tokens[i:i + (1 << 17)].long()])


def test_head_gradients_of_many_states():
    import torch
    import paper_2506_06122_amd as R
    torch.manual_seed(3)
    rows, vocab, hidden = (1 << 20) + 5, 256, 4096
    h = torch.empty(rows, hidden, device="cuda", dtype=torch.bfloat16).normal_()
    w = (torch.randn(vocab, hidden, device="cuda") / 64).bfloat16()
    t = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32)
    g = torch.randn(rows, device="cuda")
    g[::3] = 0
    logp, ent, stats = R.rollout_head_logprobs(h, w, t)
    dh, dw = R.rollout_head_logprobs_grad(h, w, t, stats, ent, g)
    assert not dh[::3].any()
    for at in (0, rows // 2, rows - 500):
        s = slice(at, at + 500)
        p = torch.softmax(h[s].double() @ w.double().T, 1)
        d = -p * g[s, None]
        d.scatter_add_(1, t[s].long()[:, None], g[s, None].double())
        want = d @ w.double()
        # two roundings to bf16, each at most 2^-8 relative to its value: their norms add up to less than 2^-7
        assert float((dh[s].double() - want).norm() / want.norm()) <= 2 * BF
    total = torch.zeros(vocab, hidden, device="cuda", dtype=torch.float64)
    for at in range(0, rows, 1 << 17):
        s = slice(at, at + (1 << 17))
        p = torch.softmax(h[s].double() @ w.double().T, 1)
        d = -p * g[s, None]
        d.scatter_add_(1, t[s].long()[:, None], g[s, None].double())
        total += d.T.contiguous() @ h[s].double()
    assert float((dw.double() - total).norm() / total.norm()) <= 2 * BF


def test_equal_greatest_values_in_the_longest_rows():
    """One greatest value in each of a workgroup's 4 x 256 runs of vectors, at either end of it."""
    import torch
    import paper_2506_06122_amd as R
    rows, vocab = 1024, 1 << 24
    steps = vocab // 8 // 1024
    x = torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)
    run, thread = torch.meshgrid(torch.arange(4), torch.arange(256), indexing="ij")
    step = torch.where((run + thread) % 2 == 0, 0, steps - 1)
    where = (((run * steps + step) * 256 + thread) * 8 + thread % 8).flatten()
    x.index_fill_(1, where.cuda(), 1.0)
    logp, ent, stats, ids, alt = R.rollout_token_logprobs(x, top=64)
    first = where.sort().values[:64].int().cuda()
    assert bool((ids == first).all())
    # ln(1024 e + (2^24 - 1024)) - 1, summed in 2^11 or so steps a thread and then joined
    import math
    log_s = math.log(1024 + (vocab - 1024) / math.e)
    assert float((stats[:, 1].double() - log_s).abs().max()) <= (vocab // 256) * U
    assert float((alt.double() + log_s).abs().max()) <= (vocab // 256) * U


def test_gradient_of_a_matrix_past_32_gb():
    import torch
    import paper_2506_06122_amd as R
    torch.manual_seed(5)
    vocab, hidden, n = 1 << 22, 4160, 3000  # 35 GB
    ids = torch.randint(0, vocab, (n,), device="cuda", dtype=torch.int32)
    ids[:5] = torch.tensor([vocab - 1, 0, 17, vocab - 1, vocab])
    dy = torch.randn(n, hidden, device="cuda").bfloat16()
    out = torch.full((vocab, hidden), 1.0, dtype=torch.bfloat16, device="cuda")
    R.rollout_embed_grad(dy, ids, vocab, out=out)
    inside = ids < vocab
    rows, at = ids[inside].long().unique(return_inverse=True)
    want = torch.zeros(len(rows), hidden, device="cuda", dtype=torch.float64).index_add_(0, at, dy[inside].double())
    got = out[rows]
    # few rows to an id: the sum's roundings are far below half a step of bf16
    assert float(((got.double() - want).abs() - BF * 1.001 * want.abs()).max()) <= 1e-6
    out[rows] = 0
    for i in range(0, vocab, 1 << 19):
        assert not out[i:i + (1 << 19)].any()


@pytest.mark.parametrize("vocab,pad", [(152064, 0), (152063, 2)])
def test_logits_past_the_last_cache(vocab, pad):
    import math
    import torch
    import paper_2506_06122_amd as R
    torch.manual_seed(6)
    rows = 1100  # 335 MB
    buf = torch.empty(rows, vocab + pad, device="cuda", dtype=torch.bfloat16).normal_(0, 3)
    x = buf[:, pad:]
    x[7] = -math.inf
    x[8, 1000:] = -math.inf
    t = torch.randint(-1, vocab, (rows,), device="cuda", dtype=torch.int32)
    lp = torch.log_softmax(x.double(), 1)
    want = torch.where(t >= 0, lp.gather(1, t.clamp(min=0).long()[:, None])[:, 0], 0.0)
    ent = -(lp.exp() * lp.clamp(min=-1e9)).sum(1)
    ent[7] = 0
    want[7] = -math.inf if int(t[7]) >= 0 else 0.0
    live = torch.ones(rows, dtype=torch.bool, device="cuda")
    live[7] = False
    # sums of vocab / 256 values a thread, the threads' below each other, exponents of up to 2 x 30
    n = vocab / 256 + 60
    for top in (0, 5):
        logp, h, stats, ids, alt = R.rollout_token_logprobs(x, t, top=top)
        held = live & torch.isfinite(want)
        assert bool((logp == want)[~held].all())
        # |logp| <= 40: its two differences round by 4 U of that
        assert float((logp - want).abs()[held].max()) <= (n + 8) * U + 4 * U * 40
        assert float((h - ent).abs().max()) <= (3 * n + 40) * U * math.log(vocab + 2)
        if top:
            best = x.double().topk(top, 1).values
            assert bool((x.double().gather(1, ids.long()) == best)[live].all())
            assert float((alt - (lp.gather(1, ids.long())))[live].abs().max()) <= (n + 8) * U + 4 * U * 40
