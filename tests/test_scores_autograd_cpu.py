"""What the loss's backward pass hands to its kernel, on the CPU: the launches are stand-ins that look
at their arguments only."""
import pytest
import torch

sc = pytest.importorskip("paper_1111_1373_amd.scores", reason="libdscores.so not built")


class _Here:
    def __init__(self, x, stream, inputs):
        pass

    def __enter__(self):
        return 0

    def __exit__(self, *exc):
        return False


@pytest.fixture
def calls(monkeypatch):
    """(row arguments, teacher's values, index, stats) of every backward launch."""
    seen = []

    def rows_of(x, votes):
        n, classes = x.shape
        assert classes == 1 or x.stride(1) == 1
        return x.data_ptr(), 0, n, classes, x.stride(0)

    def loss(rows, x, values, index, k, temperature, g, grad, ld_grad, s):
        return x.detach().sum(1), torch.zeros(x.shape[0], 2)

    def gradient(rows, values, index, k, temperature, stats, g, grad, ld_grad, s):
        seen.append((rows, values, index, stats))
        grad.zero_()

    monkeypatch.setattr(sc, "_scores_arg", rows_of)
    monkeypatch.setattr(sc, "_On", _Here)
    monkeypatch.setattr(sc, "_loss", loss)
    monkeypatch.setattr(sc, "_gradient", gradient)
    return seen


def _inputs(n=5, classes=7, k=2):
    return (torch.randn(n, classes), torch.randn(n, k),
            torch.zeros(n, k, dtype=torch.int32))


def test_scores_where_they_were(calls):
    base, values, index = _inputs(classes=9)
    x = base[:, 2:].detach().requires_grad_()
    sc.distill_loss(x, values, index, 2.0).sum().backward()
    (rows, *_), = calls
    assert rows == (x.data_ptr(), 0, 5, 7, 9)


@pytest.mark.parametrize("how", ["clone", "wider", "transposed"])
def test_saved_scores_that_come_back_elsewhere(calls, how):
    """The place and the strides are those of the tensor that was unpacked."""
    x, values, index = _inputs()
    x.requires_grad_()
    came = []

    def unpack(t):
        if t.shape == x.shape:
            if how == "clone":
                t = t.clone()
            elif how == "wider":
                t = torch.cat([t, t], 1)[:, : t.shape[1]]
            else:
                t = t.t().contiguous().t()
            came.append(t)
        return t

    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.clone(), unpack):
        loss = sc.distill_loss(x, values, index)
    loss.sum().backward()
    (rows, *_), = calls
    assert rows[0] != x.data_ptr()
    if how == "transposed":         # rows that no kernel takes are laid out first
        assert rows[2:] == (5, 7, 7)
    else:
        assert (rows[0], *rows[2:]) == (came[-1].data_ptr(), 5, 7, came[-1].stride(0))


def test_teacher_that_comes_back_elsewhere(calls):
    x, values, index = _inputs()
    x.requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(
            lambda t: t, lambda t: t if t.shape == x.shape else t.t().contiguous().t()):
        loss = sc.distill_loss(x, values, index)
    loss.sum().backward()
    (_, v, i, stats), = calls
    assert v.is_contiguous() and i.is_contiguous() and stats.is_contiguous()


@pytest.mark.parametrize("wrong", ["float64", "long", "shorter"])
def test_saved_tensors_of_another_kind_are_refused(calls, wrong):
    x, values, index = _inputs()
    x.requires_grad_()

    def unpack(t):
        if wrong == "float64" and t.dtype == torch.float32 and t.shape == values.shape:
            return t.double()
        if wrong == "long" and t.dtype == torch.int32:
            return t.long()
        if wrong == "shorter" and t.dtype == torch.int32:
            return t[:3]
        return t

    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        loss = sc.distill_loss(x, values, index)
    with pytest.raises(ValueError):
        loss.sum().backward()
    assert not calls


def test_under_checkpoint(calls):
    """The scores of the first forward pass are gone; the recomputed ones are used."""
    from torch.utils.checkpoint import checkpoint
    h, values, index = _inputs(classes=4)
    w = torch.randn(4, 7, requires_grad=True)
    made, keep = [], []

    def head(h):
        x = h @ w
        made.append(x.data_ptr())
        keep.append(torch.empty_like(x))        # takes another place between the passes
        return sc.distill_loss(x, values, index, 1.5)

    loss = checkpoint(head, h, use_reentrant=False)
    keep.append(torch.empty(5, 7))
    loss.sum().backward()
    (rows, *_), = calls
    assert len(made) == 2 and rows[0] == made[1]
