"""What the calls at the vocabulary's ends promise of memory: a workspace's contents mean nothing, and only the results are written -
not the inputs, not what lies around any array."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
GUARD = 4096


class Arrays:
    """Arrays of one call in one buffer, guards between them."""

    def __init__(self, fill):
        self.fill, self.at, self.parts = fill, GUARD, []

    def take(self, name, shape, dtype, values=None, odd=0):
        """`odd`: elements past an aligned address."""
        size = dtype.itemsize
        self.at = (self.at + 255) // 256 * 256 + odd * size
        self.parts.append((name, self.at, tuple(shape), dtype, values))
        self.at += int(np.prod(shape)) * size + GUARD
        return name

    def place(self):
        import torch
        self.buf = torch.full((self.at + GUARD,), self.fill, dtype=torch.uint8, device="cuda")
        out = {}
        for name, at, shape, dtype, values in self.parts:
            n = int(np.prod(shape)) * dtype.itemsize
            out[name] = self.buf[at:at + n].view(dtype).view(shape)
            if values is not None:
                out[name].copy_(values)
        self.before = self.buf.clone()
        return out

    def check(self, written):
        import torch
        same = self.buf == self.before
        for name, at, shape, dtype, _ in self.parts:
            if name in written:
                same[at:at + int(np.prod(shape)) * dtype.itemsize] = True
        assert bool(same.all()), torch.nonzero(~same).flatten()[:8].tolist()


def run(call, fill):
    """call(arrays) -> (name, arguments with names of arrays, sizes of the workspace, results); the results' bits."""
    import torch
    from paper_2506_06122_amd import binding as B
    lib = B.load_library()
    a = Arrays(fill)
    name, args, sizes, results = call(a)
    need = getattr(lib, name + "_workspace")(*sizes) if sizes else 0
    assert need >= 0
    a.take("workspace", (max(need, 1),), torch.uint8)
    t = a.place()
    values = [t[x].data_ptr() if isinstance(x, str) else x for x in args]
    at = args.index("workspace") + 1 if "workspace" in args else None
    if at:
        values[at] = need
    assert getattr(lib, name)(*values) == B.OK, lib.rollout_last_error(None)
    torch.cuda.synchronize()
    a.check(set(results) | {"workspace"})
    return [t[r].clone().view(torch.uint8) for r in results]


def same_whatever_was_there(call):
    import torch
    first = None
    for fill in (0xff, 0x00, 0x7b):
        got = run(call, fill)
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(first, got))


def random(shape, dtype, seed, spread=1.0):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (torch.randn(*shape, device="cuda", generator=gen) * spread).to(dtype)


def ids(n, vocab, seed):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randint(-1, vocab + 1, (n,), device="cuda", dtype=torch.int32, generator=gen)


@pytest.mark.parametrize("rows,vocab,top,odd", [(1, 151936, 20, 0), (3, 50257, 64, 1), (70, 5003, 5, 3), (600, 1999, 0, 0), (2, 1, 1, 1)])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_logprobs_and_their_gradient(rows, vocab, top, odd, dtype):
    import torch
    kind = [torch.float32, torch.bfloat16, torch.float16][dtype]

    def forward(a):
        a.take("x", (rows, vocab), kind, random((rows, vocab), kind, 1, 2.5), odd)
        a.take("t", (rows,), torch.int32, ids(rows, vocab, 2))
        for n in ("logp", "entropy"):
            a.take(n, (rows,), torch.float32)
        a.take("stats", (rows, 2), torch.float32)
        a.take("top_ids", (rows, max(top, 1)), torch.int32)
        a.take("top_logp", (rows, max(top, 1)), torch.float32)
        return ("rollout_token_logprobs", ["x", dtype, rows, vocab, vocab, 0.8, "t", top, "workspace", 0, None, "logp", "entropy", "stats",
                                           "top_ids", "top_logp"], (rows, vocab, top),
                ["logp", "entropy", "stats"] + (["top_ids", "top_logp"] if top else []))

    def backward(a):
        import paper_2506_06122_amd as R
        x, t = random((rows, vocab), kind, 1, 2.5), ids(rows, vocab, 2)
        _, entropy, stats, _, _ = R.rollout_token_logprobs(x, t, temperature=0.8)
        a.take("x", (rows, vocab), kind, x, odd)
        a.take("t", (rows,), torch.int32, t)
        a.take("stats", (rows, 2), torch.float32, stats)
        a.take("entropy", (rows,), torch.float32, entropy)
        a.take("g", (rows,), torch.float32, random((rows,), torch.float32, 3))
        a.take("h", (rows,), torch.float32, random((rows,), torch.float32, 4, 0.1))
        a.take("out", (rows, vocab), kind, None, odd // 2)
        return ("rollout_token_logprobs_grad", ["x", dtype, rows, vocab, vocab, 0.8, "t", "stats", "entropy", "g", "h", None, "out", vocab], None, ["out"])

    same_whatever_was_there(forward)
    same_whatever_was_there(backward)


@pytest.mark.parametrize("n,vocab,hidden,odd", [(1, 7, 64, 0), (1021, 300, 128, 0), (5000, 2003, 96, 0), (333, 50, 33, 1), (4100, 3, 512, 0)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_embedding_and_its_gradient(n, vocab, hidden, odd, dtype):
    import torch
    kind = [torch.float32, torch.bfloat16][dtype]

    def lookup(a):
        a.take("table", (vocab, hidden), kind, random((vocab, hidden), kind, 1), odd)
        a.take("t", (n,), torch.int32, ids(n, vocab, 2))
        a.take("out", (n, hidden), kind, None, odd)
        return "rollout_embed", ["table", dtype, vocab, hidden, hidden, "t", n, 1.5, None, "out"], None, ["out"]

    def gradient(base):
        def call(a):
            a.take("dy", (n, hidden), kind, random((n, hidden), kind, 3), odd)
            a.take("t", (n,), torch.int32, ids(n, vocab, 2))
            if base:
                a.take("base", (vocab, hidden), torch.float32, random((vocab, hidden), torch.float32, 4), odd)
            a.take("out", (vocab, hidden), torch.float32, None, odd)
            return ("rollout_embed_grad", ["dy", dtype, n, vocab, hidden, hidden, "t", 1.5, "base" if base else None, 0, "workspace", 0, None, "out"],
                    (n, vocab, hidden), ["out"])
        return call

    def in_place(a):
        a.take("dy", (n, hidden), kind, random((n, hidden), kind, 3), odd)
        a.take("t", (n,), torch.int32, ids(n, vocab, 2))
        a.take("out", (vocab, hidden), torch.float32, random((vocab, hidden), torch.float32, 4), odd)
        return ("rollout_embed_grad", ["dy", dtype, n, vocab, hidden, hidden, "t", 1.5, "out", 0, "workspace", 0, None, "out"], (n, vocab, hidden), ["out"])

    for call in (lookup, gradient(False), gradient(True), in_place):
        same_whatever_was_there(call)


@pytest.mark.parametrize("rows,vocab,hidden", [(1, 7, 64), (7, 50257, 128), (40, 1031, 320), (100, 50257, 64), (130, 1031, 256), (300, 32001, 64),
                                               (613, 5003, 192), (1500, 12301, 64)])
def test_lm_head(rows, vocab, hidden):
    import torch
    import paper_2506_06122_amd as R
    bf = torch.bfloat16
    h, w, t = random((rows, hidden), bf, 1), random((vocab, hidden), bf, 2, 0.3), ids(rows, vocab, 3)
    _, entropy, stats = R.rollout_head_logprobs(h, w, t, temperature=0.9)
    g, e = random((rows,), torch.float32, 4), random((rows,), torch.float32, 5, 0.1)
    g[::3] = e[::3] = 0

    def inputs(a):
        a.take("h", (rows, hidden), bf, h)
        a.take("w", (vocab, hidden), bf, w)
        a.take("t", (rows,), torch.int32, t)

    def forward(a):
        inputs(a)
        for n in ("logp", "entropy"):
            a.take(n, (rows,), torch.float32)
        a.take("stats", (rows, 2), torch.float32)
        return ("rollout_head_logprobs", ["h", hidden, "w", hidden, rows, vocab, hidden, 0.9, "t", "workspace", 0, None, "logp", "entropy", "stats"],
                (rows, vocab, hidden), ["logp", "entropy", "stats"])

    def backward(a):
        inputs(a)
        a.take("stats", (rows, 2), torch.float32, stats)
        a.take("entropy", (rows,), torch.float32, entropy)
        a.take("g", (rows,), torch.float32, g)
        a.take("e", (rows,), torch.float32, e)
        a.take("dh", (rows, hidden), bf)
        a.take("dw", (vocab, hidden), bf)
        return ("rollout_head_logprobs_grad", ["h", hidden, "w", hidden, rows, vocab, hidden, 0.9, "t", "stats", "entropy", "g", "e", "workspace", 0, None,
                                               "dh", "dw"], (rows, vocab, hidden), ["dh", "dw"])

    same_whatever_was_there(forward)
    same_whatever_was_there(backward)
