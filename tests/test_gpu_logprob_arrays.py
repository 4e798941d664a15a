"""Which arrays the gradient of logits may be written to."""
import numpy as np
import pytest

from test_gpu_token_logprobs import cuda, grads_of, make, targets_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2, 5])
def test_a_result_that_begins_where_the_logits_do_needs_their_stride(rows):
    import torch
    import paper_2506_06122_amd as R
    from paper_2506_06122_amd.binding import E_INVAL
    vocab, stride = 501, 640
    wide = torch.full((rows, stride), 7.0, device="cuda")
    x = wide[:, :vocab]
    x.copy_(torch.from_numpy(make("plain", rows, vocab, 3)))
    t = cuda(targets_of(rows, vocab, 3))
    got = R.rollout_token_logprobs(x, t)
    g, h = map(cuda, grads_of(rows, 3, True))
    held = wide.clone()
    for other in (wide.view(-1)[:rows * vocab].view(rows, vocab),                   # without the gaps
                  wide.view(-1).as_strided((rows, vocab), (vocab + 1, 1))):
        with pytest.raises(R.RolloutError) as e:
            R.rollout_token_logprobs_grad(x, t, got[2], got[1], g, h, out=other)
        assert e.value.code == E_INVAL
        assert torch.equal(wide, held)
    want = R.rollout_token_logprobs_grad(x, t, got[2], got[1], g, h)
    out = R.rollout_token_logprobs_grad(x, t, got[2], got[1], g, h, out=wide[:, :vocab])  # another view of the same rows
    assert torch.equal(out, want) and torch.equal(x, want) and bool((wide[:, vocab:] == 7.0).all())


def test_one_row_in_place_has_no_stride_of_its_own():
    import torch
    import paper_2506_06122_amd as R
    vocab = 333
    wide = torch.from_numpy(make("plain", 2, vocab + 7, 5)).cuda()
    x = wide[:1, :vocab]
    t = cuda(np.array([5], np.int32))
    got = R.rollout_token_logprobs(x, t)
    g, h = map(cuda, (np.array([1.5], np.float32), np.array([0.1], np.float32)))
    want = R.rollout_token_logprobs_grad(x, t, got[2], got[1], g, h)
    rest = wide.clone()
    out = R.rollout_token_logprobs_grad(x, t, got[2], got[1], g, h, out=wide.view(-1)[:vocab].view(1, vocab))
    assert torch.equal(out, want)
    assert torch.equal(wide[0, vocab:], rest[0, vocab:]) and torch.equal(wide[1], rest[1])
