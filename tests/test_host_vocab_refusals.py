"""What the calls at the vocabulary's ends refuse, without a GPU: every check stands before the first launch."""
import ctypes as C

import pytest
import torch

import paper_2506_06122_amd as R
from paper_2506_06122_amd import binding as B

ARRAY, OTHER, THIRD, FOURTH = (k << 24 for k in (1, 2, 3, 4))  # aligned addresses, far apart, that are never read


def call(name, args, **changed):
    values = dict(args)
    for k in changed:
        assert k in values, k
    values.update(changed)
    lib = B.load_library()
    rc = getattr(lib, name)(*values.values())
    return rc, lib.rollout_last_error(None).decode()


TOKENS = dict(logits=ARRAY, dtype=1, rows=3, vocab=100, row_stride=100, temperature=1.0, targets=ARRAY, top=4,
              workspace=None, workspace_bytes=0, stream=None, logp=ARRAY, entropy=ARRAY, row_stats=ARRAY, top_ids=ARRAY,
              top_logp=ARRAY)
GRAD = dict(logits=ARRAY, dtype=1, rows=3, vocab=100, row_stride=100, temperature=1.0, targets=ARRAY, row_stats=ARRAY,
            entropy=ARRAY, grad_logp=ARRAY, grad_entropy=ARRAY, stream=None, grad_logits=OTHER, grad_row_stride=100)
EMBED = dict(table=ARRAY, dtype=1, vocab=100, hidden=64, table_stride=64, tokens=ARRAY, n=3, scale=1.0, stream=None, out=OTHER)
EMBED_GRAD = dict(grad_rows=ARRAY, dtype=1, n=3, vocab=100, hidden=64, row_stride=64, tokens=ARRAY, scale=1.0, base=None,
                  table_dtype=1, workspace=ARRAY, workspace_bytes=1 << 20, stream=None, grad_table=OTHER)

HEAD = dict(hidden_states=ARRAY, hidden_stride=64, lm_head=ARRAY, head_stride=64, rows=3, vocab=100, hidden=64, temperature=1.0,
            targets=ARRAY, workspace=ARRAY, workspace_bytes=1 << 20, stream=None, logp=ARRAY, entropy=ARRAY, row_stats=ARRAY)
HEAD_GRAD = dict(hidden_states=ARRAY, hidden_stride=64, lm_head=OTHER, head_stride=64, rows=3, vocab=100, hidden=64,
                 temperature=1.0, targets=ARRAY, row_stats=ARRAY, entropy=ARRAY, grad_logp=ARRAY, grad_entropy=ARRAY,
                 workspace=ARRAY, workspace_bytes=1 << 20, stream=None, grad_hidden=THIRD, grad_head=FOURTH)


@pytest.mark.parametrize("name,args,changed,word", [
    ("rollout_token_logprobs", TOKENS, dict(logits=None), "logits"),
    ("rollout_token_logprobs", TOKENS, dict(logits=ARRAY + 1), "aligned"),
    ("rollout_token_logprobs", TOKENS, dict(dtype=3), "dtype"),
    ("rollout_token_logprobs", TOKENS, dict(dtype=-1), "dtype"),
    ("rollout_token_logprobs", TOKENS, dict(rows=-1), "rows"),
    ("rollout_token_logprobs", TOKENS, dict(rows=(1 << 24) + 1), "rows"),
    ("rollout_token_logprobs", TOKENS, dict(vocab=0), "vocab"),
    ("rollout_token_logprobs", TOKENS, dict(row_stride=99), "row_stride"),
    ("rollout_token_logprobs", TOKENS, dict(top=65), "top"),
    ("rollout_token_logprobs", TOKENS, dict(top=-1), "top"),
    ("rollout_token_logprobs", TOKENS, dict(vocab=3), "top"),
    ("rollout_token_logprobs", TOKENS, dict(top_ids=None), "top_ids"),
    ("rollout_token_logprobs", TOKENS, dict(top_logp=None), "top_logp"),
    ("rollout_token_logprobs", TOKENS, dict(logp=None), "logp"),
    ("rollout_token_logprobs", TOKENS, dict(entropy=None), "entropy"),
    ("rollout_token_logprobs", TOKENS, dict(row_stats=None), "row_stats"),
    ("rollout_token_logprobs", TOKENS, dict(targets=ARRAY + 2), "targets"),
    ("rollout_token_logprobs", TOKENS, dict(temperature=0.0), "temperature"),
    ("rollout_token_logprobs", TOKENS, dict(temperature=-1.0), "temperature"),
    ("rollout_token_logprobs", TOKENS, dict(temperature=float("nan")), "temperature"),
    ("rollout_token_logprobs", TOKENS, dict(temperature=float("inf")), "temperature"),
    ("rollout_token_logprobs", TOKENS, dict(temperature=1e-45), "temperature"),
    ("rollout_token_logprobs", TOKENS, dict(vocab=50000, row_stride=50000), "workspace"),
    ("rollout_token_logprobs", TOKENS, dict(vocab=50000, row_stride=50000, workspace=ARRAY + 8, workspace_bytes=1 << 20), "aligned"),
    ("rollout_token_logprobs_grad", GRAD, dict(logits=None), "logits"),
    ("rollout_token_logprobs_grad", GRAD, dict(grad_logits=None), "grad_logits"),
    ("rollout_token_logprobs_grad", GRAD, dict(grad_row_stride=99), "grad_row_stride"),
    ("rollout_token_logprobs_grad", GRAD, dict(grad_logits=ARRAY, grad_row_stride=101), "in place"),
    ("rollout_token_logprobs_grad", GRAD, dict(grad_logits=ARRAY + 2), "overlap"),
    ("rollout_token_logprobs_grad", GRAD, dict(grad_logits=ARRAY + 400, grad_row_stride=150), "overlap"),
    ("rollout_token_logprobs_grad", GRAD, dict(row_stride=200, grad_row_stride=200, grad_logits=ARRAY + 2 * 99), "overlap"),
    ("rollout_token_logprobs_grad", GRAD, dict(row_stride=200, grad_row_stride=200, grad_logits=ARRAY + 2 * 101), "overlap"),
    ("rollout_token_logprobs_grad", GRAD, dict(row_stats=None), "row_stats"),
    ("rollout_token_logprobs_grad", GRAD, dict(grad_logp=None), "grad_logp"),
    ("rollout_token_logprobs_grad", GRAD, dict(entropy=None), "entropy"),
    ("rollout_token_logprobs_grad", GRAD, dict(dtype=7), "dtype"),
    ("rollout_token_logprobs_grad", GRAD, dict(temperature=0.0), "temperature"),
    ("rollout_embed", EMBED, dict(table=None), "table"),
    ("rollout_embed", EMBED, dict(tokens=None), "tokens"),
    ("rollout_embed", EMBED, dict(out=None), "out"),
    ("rollout_embed", EMBED, dict(hidden=0), "hidden"),
    ("rollout_embed", EMBED, dict(table_stride=63), "table_stride"),
    ("rollout_embed", EMBED, dict(scale=float("inf")), "scale"),
    ("rollout_embed", EMBED, dict(n=-1), "rows"),
    ("rollout_embed", EMBED, dict(out=ARRAY + 2 * 64 * 99), "overlap"),
    ("rollout_embed", EMBED, dict(n=1 << 24, hidden=1 << 20, table_stride=1 << 20), "2^38"),
    ("rollout_embed_grad", EMBED_GRAD, dict(base=OTHER + 2), "overlap"),
    ("rollout_embed_grad", EMBED_GRAD, dict(grad_rows=OTHER + 128), "overlap"),
    ("rollout_embed_grad", EMBED_GRAD, dict(grad_rows=None), "grad_rows"),
    ("rollout_embed_grad", EMBED_GRAD, dict(tokens=None), "tokens"),
    ("rollout_embed_grad", EMBED_GRAD, dict(grad_table=None), "grad_table"),
    ("rollout_embed_grad", EMBED_GRAD, dict(table_dtype=2), "table_dtype"),
    ("rollout_embed_grad", EMBED_GRAD, dict(scale=float("nan")), "scale"),
    ("rollout_embed_grad", EMBED_GRAD, dict(row_stride=3), "row_stride"),
    ("rollout_embed_grad", EMBED_GRAD, dict(workspace_bytes=16), "workspace"),
    ("rollout_embed_grad", EMBED_GRAD, dict(workspace=None), "workspace"),
    ("rollout_embed_grad", EMBED_GRAD, dict(base=ARRAY + 1), "base"),
    ("rollout_head_logprobs", HEAD, dict(hidden_states=None), "hidden_states"),
    ("rollout_head_logprobs", HEAD, dict(hidden_states=ARRAY + 8), "aligned"),
    ("rollout_head_logprobs", HEAD, dict(lm_head=None), "lm_head"),
    ("rollout_head_logprobs", HEAD, dict(lm_head=ARRAY + 2), "aligned"),
    ("rollout_head_logprobs", HEAD, dict(hidden=96, hidden_stride=96, head_stride=96), "multiple of 64"),
    ("rollout_head_logprobs", HEAD, dict(hidden_stride=68), "hidden_stride"),
    ("rollout_head_logprobs", HEAD, dict(hidden_stride=56), "hidden_stride"),
    ("rollout_head_logprobs", HEAD, dict(head_stride=(1 << 22) + 8), "head_stride"),
    ("rollout_head_logprobs", HEAD, dict(workspace_bytes=64), "workspace"),
    ("rollout_head_logprobs", HEAD, dict(workspace=ARRAY + 4), "aligned"),
    ("rollout_head_logprobs", HEAD, dict(temperature=0.0), "temperature"),
    ("rollout_head_logprobs", HEAD, dict(vocab=0), "vocab"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(hidden_states=None), "hidden_states"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(hidden_states=ARRAY + 8), "aligned"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(lm_head=None), "lm_head"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(lm_head=ARRAY + 2), "aligned"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(hidden=96, hidden_stride=96, head_stride=96), "multiple of 64"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(hidden_stride=68), "hidden_stride"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(hidden_stride=56), "hidden_stride"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(head_stride=(1 << 22) + 8), "head_stride"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(workspace_bytes=64), "workspace"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(workspace=ARRAY + 4), "aligned"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(temperature=0.0), "temperature"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(vocab=0), "vocab"),
    ("rollout_head_logprobs", HEAD, dict(logp=None), "logp"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(grad_hidden=None), "grad_hidden"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(grad_head=ARRAY + 8), "aligned"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(entropy=None), "entropy"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(grad_head=OTHER), "overlap"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(grad_hidden=ARRAY), "overlap"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(grad_hidden=FOURTH + 64 * 99 * 2), "overlap"),
    ("rollout_head_logprobs", HEAD, dict(rows=1 << 24, vocab=1 << 24), "2^42"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(grad_logp=None), "grad_logp"),
])
def test_refused(name, args, changed, word):
    rc, text = call(name, args, **changed)
    assert rc == B.E_INVAL and word in text, (rc, text)


def test_nothing_to_do_is_done():
    assert call("rollout_token_logprobs", TOKENS, rows=0, logits=None, logp=None)[0] == 0
    assert call("rollout_token_logprobs_grad", GRAD, rows=0, logits=None)[0] == 0
    assert call("rollout_embed", EMBED, n=0, out=None)[0] == 0
    assert call("rollout_head_logprobs", HEAD, rows=0, hidden_states=None)[0] == 0


def test_workspace_sizes():
    lib = B.load_library()
    assert lib.rollout_token_logprobs_workspace(4096, 152064, 8) == 0   # a row to a workgroup
    assert lib.rollout_token_logprobs_workspace(1, 152064, 8) > lib.rollout_token_logprobs_workspace(1, 152064, 0) > 0
    assert lib.rollout_token_logprobs_workspace(1, 152064, 65) == B.E_INVAL
    assert lib.rollout_token_logprobs_workspace(-1, 152064, 0) == B.E_INVAL
    assert lib.rollout_embed_grad_workspace(100, 0, 64) == B.E_INVAL
    assert lib.rollout_embed_grad_workspace(0, 100, 64) >= 0


@pytest.mark.parametrize("bad", ["cpu"])
def test_the_binding_takes_gpu_tensors(bad):
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    for f in (lambda: R.rollout_token_logprobs(x, t), lambda: R.rollout_token_logprobs_grad(x, t, x[:, :2], x[:, 0], x[:, 0]),
              lambda: R.rollout_embed(x, t), lambda: R.rollout_embed_grad(x, t, 4),
              lambda: R.rollout_head_logprobs(x, x, t), lambda: R.rollout_head_logprobs_grad(x, x, t, x[:, :2], x[:, 0], x[:, 0])):
        with pytest.raises(R.RolloutError) as e:
            f()
        assert e.value.code == B.E_INVAL


@pytest.mark.parametrize("name,args,changed,word", [
    ("rollout_token_logprobs", TOKENS, dict(rows=(1 << 24) - 63), "2^24 - 64"),
    ("rollout_token_logprobs_grad", GRAD, dict(rows=(1 << 24) - 63), "2^24 - 64"),
    ("rollout_head_logprobs", HEAD, dict(rows=(1 << 24) - 63), "2^24 - 64"),
    ("rollout_head_logprobs_grad", HEAD_GRAD, dict(rows=(1 << 24) - 63), "2^24 - 64"),
    ("rollout_token_logprobs", TOKENS, dict(row_stride=(1 << 36) + 1), "2^36"),
    ("rollout_embed", EMBED, dict(table_stride=(1 << 36) + 1), "2^36"),
    ("rollout_embed_grad", EMBED_GRAD, dict(row_stride=(1 << 36) + 1), "2^36"),
])
def test_refused_past_the_limits(name, args, changed, word):
    rc, text = call(name, args, **changed)
    assert rc == B.E_INVAL and word in text, (rc, text)
