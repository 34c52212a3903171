"""A forest's votes (DT_OUT_VOTES_U8), and what is made of them: teacher, sampler, student."""
import numpy as np
import pytest

import oracle
from paper_1111_1373_amd import workloads as W
from tests import scoreutil as SU

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dt():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1111_1373_amd import dtree
    return dtree


def _votes(nodes, offsets, x, F, C):
    v = np.zeros((len(x), C), dtype=np.uint8)
    for a, b in zip(offsets[:-1], offsets[1:]):
        v[np.arange(len(x)), oracle.tree_classes(nodes[a:b], x, F)] += 1
    return v


def _forest(n_trees, F, C, seed):
    rng = np.random.default_rng(seed)
    trees = [W.random_full_tree(rng, int(rng.integers(1, 60)), F, C) for _ in range(n_trees)]
    return np.concatenate(trees), np.cumsum([0] + [len(t) for t in trees])


@pytest.mark.parametrize("algo", ["data", "speculative"])
@pytest.mark.parametrize("n,F,C,trees", [(1, 3, 2, 1), (63, 4, 7, 5), (64, 8, 8, 32), (1000, 19, 5, 255),
                                         (20_001, 32, 9, 20), (5_003, 33, 16, 11), (777, 70, 63, 40),
                                         (3000, 6, 64, 100), (500, 5, 1, 9)])
def test_votes(dt, n, F, C, trees, algo):
    nodes, offsets = _forest(trees, F, C, n)
    x = np.random.default_rng(n).standard_normal((n, F)).astype(np.float32)
    f = dt.Forest(nodes, offsets, F, C)
    print("votes", n, F, C, trees, algo, flush=True)
    base = torch.full((n * C + 64,), 201, dtype=torch.uint8, device="cuda")
    out = base[:n * C].view(n, C)
    f.classify(torch.from_numpy(x).cuda(), algo=algo, out_kind="votes_u8", out=out)
    want = _votes(nodes, offsets, x, F, C)
    np.testing.assert_array_equal(out.cpu().numpy(), want)
    assert (base[n * C:] == 201).all()
    # the majority of these is what the forest answers
    np.testing.assert_array_equal(f.classify(torch.from_numpy(x).cuda(), algo=algo).cpu().numpy(),
                                  np.argmax(want, 1))
    off = base[1:1 + n * C].view(n, C)              # rows that start between words
    f.classify(torch.from_numpy(x).cuda(), algo=algo, out_kind="votes_u8", out=off)
    np.testing.assert_array_equal(off.cpu().numpy(), want)


def test_votes_in_a_hip_graph(dt):
    nodes, offsets = _forest(30, 12, 10, 3)
    xs = [np.random.default_rng(i).standard_normal((9000, 12)).astype(np.float32) for i in (1, 2)]
    f = dt.Forest(nodes, offsets, 12, 10)
    x = torch.from_numpy(xs[0]).cuda()
    out = f.classify(x, out_kind="votes_u8")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f.classify(x, out_kind="votes_u8", out=out)
    for rep in range(4):
        x.copy_(torch.from_numpy(xs[rep % 2]))
        out.fill_(9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(out.cpu().numpy(), _votes(nodes, offsets, xs[rep % 2], 12, 10))


def test_forest_as_a_teacher(dt):
    """Records through a forest, its votes cut to the best classes, a student's loss and gradient
    against them, and classes drawn from the votes: each step against the plain one."""
    from paper_1111_1373_amd import scores
    w = W.config(5, n_samples=3_000)
    x_np = w.features()
    C = w.n_classes
    f = dt.Forest(w.nodes, w.tree_offsets, w.n_features, C)
    x = torch.from_numpy(x_np).cuda()
    rng = np.random.default_rng(0)
    weight = torch.from_numpy((rng.standard_normal((w.n_features, C)) * 0.2).astype(np.float32)).cuda()
    weight.requires_grad_()
    u = rng.random(len(x_np)).astype(np.float32)

    votes = f.classify(x, out_kind="votes_u8")
    values, index, lse = scores.top_scores(votes, 3)
    label = scores.sample(votes, torch.from_numpy(u).cuda(), top_p=0.9)
    student = x @ weight
    loss = scores.distill_loss(student, values, index, 2.0)
    loss.mean().backward()

    want = _votes(w.nodes, w.tree_offsets, x_np, w.n_features, C)
    np.testing.assert_array_equal(votes.cpu().numpy(), want)
    wv, wi, wl = SU.top_scores(want, 3)
    np.testing.assert_array_equal(index.cpu().numpy(), wi)
    np.testing.assert_allclose(values.cpu().numpy(), wv, rtol=2.0 ** -22)
    np.testing.assert_allclose(lse.cpu().numpy(), np.log(len(w.tree_offsets) - 1.0), rtol=2.0 ** -22)
    np.testing.assert_array_equal(label.cpu().numpy(), SU.sample(want, u, top_p=0.9))
    s = student.detach().cpu().numpy()
    wloss, wgrad = SU.distill(s, values.cpu().numpy(), wi, 2.0, np.full(len(s), 1 / len(s)))
    assert np.abs(loss.detach().cpu().numpy() - wloss).max() <= 4 * (np.ptp(s) + 40) * 2.0 ** -22
    # the weights' gradient: records' gradients (each within the student's error) times records,
    # the product's own sums of n terms in 32 bits
    want_w = x_np.astype(np.float64).T @ wgrad
    tol = (np.abs(x_np).T.astype(np.float64) @ np.abs(wgrad)) * (len(s) + 64) * 2.0 ** -24
    tol += np.abs(x_np).sum(0)[:, None] * (2.0 / len(s)) * (np.ptp(s) + 40) * 2.0 ** -21
    assert (np.abs(weight.grad.cpu().numpy() - want_w) <= tol).all()
