"""The workspaces of the log probabilities from hidden states and of their gradient, against what the header says of them; calls of no groups; weights that are no matrices."""
import pytest
import torch

from paper_1805_10032_b200 import build as zbuild
from paper_1805_10032_b200 import zeno

P = 0x1000           # an address that is checked and never read
F32, BF16 = 0, 1
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    zbuild.build()
    return zeno.load_library()


def up(v, to):
    return -(-v // to) * to


# type, param_type, m, n, cols, vocab, weights of every group's own
SIZES = [(F32, F32, 21, 128, 4096, 32000, True), (F32, F32, 33, 128, 8192, 32000, True), (F32, F32, 31, 6826, 49, 21782, False), (BF16, BF16, 8, 32768, 1024, 131072, False),
         (F32, F32, 1, 1 << 20, 64, 131072, False), (F32, F32, 1, 42608, 64, 131072, False), (BF16, BF16, 1, 63999, 64, 131072, False), (BF16, F32, 1, 64, 65000, 131072, False),
         (BF16, BF16, 21, 5, 1024, 32000, True), (BF16, BF16, 2, 2048, 4096, 131072, False), (F32, F32, 3, 57, 777, 5001, False), (BF16, BF16, 1, 20, 1023, 151936, False),
         (BF16, BF16, 1, 13, 4096, 300, False), (F32, BF16, 40, 1, 264, 513, True), (F32, F32, 1, 1, 1, 1, False), (BF16, BF16, 60000, 1, 8, 30, False)]


@pytest.mark.parametrize("type,ptype,m,n,cols,vocab,models", SIZES)
def test_no_larger_than_the_header_says(lib, type, ptype, m, n, cols, vocab, models):
    ldw = vocab * cols if models else 0
    terms = 3 if F32 in (type, ptype) else 2
    x_entry, w_entry = 6 if type == F32 else 2, 6 if ptype == F32 else 2
    as_it_lies = ptype == BF16 and cols % 8 == 0
    row = up(cols, 8)
    # a word's rewritten entries, of all groups; pieces are whole tiles of 256 words
    word = 0 if as_it_lies else (m if models else 1) * row * w_entry
    weights = min(max(768 * MB, 2048 * word), up(vocab, 256) * word)
    tokens = up(m * up(n, 128 if n <= 128 else 256), 64) if models else up(m * n, 64)
    forward = weights + tokens * (row * x_entry + up(vocab, 256) // 64 * 8 + 16) + 12 * m
    assert 0 < lib.zeno_linear_logprobs_workspace(type, ptype, m, n, cols, vocab, P, ldw) <= forward + 40 * MB
    tokens = up(m * up(n, 256 if models else 16), 64)
    probs = min(max(512 * MB, 2048 * tokens * terms * 2), up(vocab, 256) * tokens * terms * 2)
    for want_dx in (0, 1):
        gradient = weights + probs + tokens * (row * x_entry + want_dx * row * 4 + 20) + 12 * m
        assert 0 < lib.zeno_linear_logprobs_gradient_workspace(type, ptype, m, n, cols, vocab, P, ldw, want_dx) <= gradient + 40 * MB


def test_no_groups_with_weights_of_their_own(lib):
    """Of no groups there are no weights, nor an address of them."""
    x = zeno.RowsDesc(None, 64, 640)
    assert lib.zeno_embed(0, F32, F32, None, 0, 10, 100, 64, None, 6400, 1.0, x, None) == zeno.OK
    assert lib.zeno_embed_gradient(0, F32, F32, None, x, 0, 10, 100, 64, 1.0, 0, None, 6400, None, 0, None) == zeno.OK
    assert lib.zeno_linear_logprobs_workspace(F32, F32, 0, 10, 64, 100, None, 6400) == 0
    assert lib.zeno_linear_logprobs(0, F32, F32, x, 0, 10, 64, 100, None, 6400, None, 1.0, None, None, None, 0, None) == zeno.OK
    assert lib.zeno_linear_logprobs_gradient_workspace(F32, F32, 0, 10, 64, 100, None, 6400, 1) == 0
    assert lib.zeno_linear_logprobs_gradient(0, F32, F32, x, 0, 10, 64, 100, None, 6400, None, 1.0, None, None, x, None, 6400, None, 0, None) == zeno.OK


def test_weights_of_one_dimension_are_refused():
    t, x, p, w = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 8), torch.zeros(2, 3), torch.zeros(8)
    for call in (lambda: zeno.embed(t, w), lambda: zeno.embed_gradient(t, x, w), lambda: zeno.linear_logprobs(x, w, t), lambda: zeno.linear_logprobs_gradient(x, w, t, p, p)):
        with pytest.raises(ValueError, match="is needed"):
            call()
