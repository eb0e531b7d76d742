"""A language model's training step through the C ABI: embedding, cells,
vocabulary head, the cells' backward, the table's gradient -- against the
oracle's softmax head over the same inputs, whose dX, summed by word, is the
table's gradient."""
import numpy as np
import pytest
import torch

import lm_ref as R
import oracle
from parity import check_fp32
from paper_1712_04048_amd import binding as B
from paper_1712_04048_amd import workloads as W
from paper_1712_04048_amd.runner import Batch, LmBatch

pytestmark = pytest.mark.gpu

KEYS = ["h", "c", "loss", "dWx", "dU", "db", "dWs", "dbs", "dE"]


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def _model(kind, C, seed, n_words=50, labels="all"):
    rng = np.random.Generator(np.random.PCG64(seed))
    if kind == "chain":
        graphs, N = [W.chain(int(n)) for n in rng.integers(5, 40, size=9)], 1
    else:
        graphs, N = [W.random_split_tree(int(n), rng) for n in rng.integers(2, 30, size=12)], 2
    wl = W.make_workload("lm_%s" % kind, graphs, N=N, D=20, H=128, C=C, sigma=0.1, rng=rng,
                         inputs="all" if kind == "chain" else "leaves", labels=labels)
    E = rng.standard_normal((n_words, wl.D)).astype(np.float32)
    words = np.minimum((n_words ** rng.random(wl.n_x) - 1).astype(np.int32), n_words - 1)
    words[::11] = -1   # places without a word: zero rows
    return wl, E, words


def _reference(wl, E, words, scale, precision):
    X = np.where((words >= 0)[:, None], E[np.maximum(words, 0)] * np.float32(scale),
                 np.float32(0)).astype(np.float32)
    r = oracle.run(wl, X=X, precision=precision)
    dE = np.zeros(E.shape)
    np.add.at(dE, words[words >= 0], r["dX"][words >= 0] * np.float64(np.float32(scale)))
    r["dE"] = dE
    return r


@pytest.mark.parametrize("kind,C,labels", [("chain", 4096, "all"), ("chain", 999, "all"),
                                           ("tree", 777, "root"), ("tree", 64, "all")])
def test_training_step_equals_the_softmax_head_s(ctx, kind, C, labels):
    wl, E, words = _model(kind, C, C, labels=labels)
    b = LmBatch(wl, torch.from_numpy(E).cuda(), words, ctx, scale=1.7)
    b.schedule()
    got = b.run()
    check_fp32(got, _reference(wl, E, words, 1.7, "f64"), _reference(wl, E, words, 1.7, "f32"), KEYS,
               "lm_%s_c%d" % (kind, C))
    assert b.run_infer()["loss"] == got["loss"]


def test_the_two_heads_agree(ctx):
    """cavs_forward's own head, which keeps the logits, and the one that does not."""
    wl, E, words = _model("chain", 1000, 5)
    b = LmBatch(wl, torch.from_numpy(E).cuda(), words, ctx)
    b.schedule()
    got = b.run()
    wl.X = b.X.cpu().numpy()
    own = Batch(wl, ctx).run()
    f64 = _reference(wl, E, words, 1.0, "f64")
    f32 = _reference(wl, E, words, 1.0, "f32")
    check_fp32(own, f64, f32, KEYS[:-1], "kept")
    check_fp32(got, f64, f32, KEYS, "not kept")


def test_distilling_step(ctx):
    """A teacher's words: the head's part against its 64-bit form on the states
    that the cells gave, and the rest of the step with its dh as dH_ext."""
    wl, E, words = _model("chain", 500, 6)
    rng = np.random.Generator(np.random.PCG64(1))
    top = rng.integers(0, 500, (wl.V, 7)).astype(np.int32)
    top[::3, 4:] = -1
    logit = (2 * rng.standard_normal((wl.V, 7))).astype(np.float32)
    b = LmBatch(wl, torch.from_numpy(E).cuda(), words, ctx, teacher=(top, logit, 0.6, 2.0))
    b.schedule()
    got = b.run()
    h = b.head
    want, bound = R.head(h.h, h.Ws, h.bs, h.label, h.top_word, h.top_logit, h.alpha, h.temp)
    far = {"loss": b.loss, "row_loss": b.row_loss, "dh": b.dH_ext, "dWs": b.grads["dWs"],
           "dbs": b.grads["dbs"]}
    assert all(R.outside(v, want[k], bound[k]) <= 1.0 for k, v in far.items())
    wl.X, wl.loss = b.X.cpu().numpy(), W.LOSS_NONE
    ext = b.dH_ext.cpu().numpy()
    check_fp32(got, oracle.run(wl, dH_ext=ext), oracle.run(wl, dH_ext=ext, precision="f32"),
               ["h", "c", "dWx", "dU", "db", "dX"], "distilling")


def test_bf16_table_and_head(ctx):
    """bf16 table and head weights around fp32 cells: the head against its
    64-bit form, the table's gradient against the sum of the step's own dX."""
    wl, E, words = _model("tree", 1201, 7)
    b = LmBatch(wl, torch.from_numpy(E).cuda().bfloat16(), words, ctx, scale=2.0,
                head_dtype=torch.bfloat16)
    b.schedule()
    b.run()
    h = b.head
    want, bound = R.head(h.h, h.Ws, h.bs, h.label)
    for k, v in (("loss", b.loss), ("dh", b.dH_ext), ("dWs", b.grads["dWs"]), ("dbs", b.grads["dbs"])):
        assert R.outside(v, want[k], bound[k]) <= 1.0, k
    dE, lim = R.embed_grad(b.words, b.grads["dX"], E.shape[0], 2.0, True)
    assert R.outside(b.grads["dE"], dE, lim) <= 1.0
    assert torch.equal(b.X, R.embed(b.emb.E, b.words, 2.0).float())


def test_captured_step_with_new_words(ctx):
    """The whole step but the schedule in one graph, replayed between eager steps."""
    wl, E, words = _model("chain", 800, 8)
    s = torch.cuda.Stream()
    own = B.Context(0, s)
    table = torch.from_numpy(E).cuda()
    b = LmBatch(wl, table, words, own)
    torch.cuda.synchronize()
    b.schedule()
    b.alloc()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.forward()
        b.backward()
    eager = LmBatch(wl, table, words, ctx)
    eager.schedule()
    rng = np.random.Generator(np.random.PCG64(2))
    for _ in range(3):
        new = torch.from_numpy(rng.integers(-1, E.shape[0], wl.n_x).astype(np.int32)).cuda()
        b.words.copy_(new)
        eager.words.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        want = eager.run()
        torch.cuda.synchronize()
        got = b.results()
        assert got["loss"] == want["loss"]
        for k in KEYS:
            assert np.array_equal(got[k], want[k]), k
    own.sync()
    own.close()
