"""When the feed-forward keeps gate and up values for a gradient, without a GPU:
the library's call is replaced by one that records what it is given."""
import pytest
import torch

from paper_2111_04867_amd import experts as X


@pytest.fixture
def kept(monkeypatch):
    """Shapes of `pre` that the calls got, or None."""
    seen = []

    def ffn_tensors(buffer, counts, w_in, w_out, out, workspace, *, pre=None, stream=None):
        seen.append(None if pre is None else tuple(pre.shape))
        out.zero_()

    monkeypatch.setattr(X, "ffn_tensors", ffn_tensors)
    return seen


def arrays(*trained):
    """Buffer, counts and weights of 3 experts, dim 8, hidden 6; those named want a gradient."""
    a = {"buffer": torch.zeros(2, 3, 5, 8), "counts": torch.zeros(2, 3, dtype=torch.int32),
         "w_in": torch.zeros(3, 12, 8), "w_out": torch.zeros(3, 8, 6)}
    for n in trained:
        a[n].requires_grad_()
    return a.values()


ALL = ("buffer", "w_in", "w_out")


@pytest.mark.parametrize("off", [torch.no_grad, torch.inference_mode])
@pytest.mark.parametrize("trained", [ALL, ("w_in", "w_out"), ("w_out",), ()], ids=str)
def test_nothing_is_kept_without_gradients(kept, off, trained):
    """Weights that are trained elsewhere do not make an evaluation store them."""
    values = arrays(*trained)
    with off():
        assert not X.ffn(*values).requires_grad
    assert kept == [None]


@pytest.mark.parametrize("trained", [ALL, ("buffer",), ("w_in",), ("w_out",)], ids=str)
def test_kept_for_a_gradient(kept, trained):
    assert X.ffn(*arrays(*trained)).requires_grad
    with torch.no_grad(), torch.enable_grad():
        X.ffn(*arrays(*trained))
    X.ffn(*arrays())
    assert kept == [(2, 3, 5, 12), (2, 3, 5, 12), None]


@pytest.mark.gpu
def test_memory_and_results_of_an_evaluation():
    """The memory of a call without gradients has no room for `pre`; its rows
    are the training pass's."""
    e, c, d, f = 4, 300, 64, 2048
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(e, c, d, generator=gen, device="cuda").half()
    counts = torch.tensor([300, 0, 7, 299], dtype=torch.int32, device="cuda")
    w_in, w_out = ((torch.randn(*s, generator=gen, device="cuda") / 8).half().requires_grad_()
                   for s in ((e, 2 * f, d), (e, d, f)))
    want = X.ffn(x, counts, w_in, w_out)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    with torch.no_grad():
        got = X.ffn(x, counts, w_in, w_out)
    used = torch.cuda.max_memory_allocated() - before
    # the allocator rounds the two arrays up to 512 bytes each, and a block for the
    # larger one keeps a rest of up to 1 MB; pre would take 4 * 300 * 2 * 2048 * 2
    # bytes, 9.8 MB
    rest = 2 * 512 + (1 << 20)
    assert used <= x.nbytes + X.ffn_workspace(x.shape, f, x.dtype) + rest
    assert torch.equal(got, want)
