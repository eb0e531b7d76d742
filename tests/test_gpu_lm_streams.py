"""A language model's steps on a stream of their own, beside work on torch's
current one."""
import numpy as np
import pytest
import torch

from paper_1712_04048_amd import binding as B
from paper_1712_04048_amd import workloads as W
from paper_1712_04048_amd.runner import LmBatch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.mark.parametrize("head_dtype", [torch.float32, torch.bfloat16])
def test_steps_on_a_stream_of_their_own(head_dtype):
    """The same bits as on torch's stream, from the first step on; small tensors
    that torch makes and fills while the steps are on their way keep their values."""
    rng = np.random.Generator(np.random.PCG64(3))
    wl = W.make_workload("lm", [W.chain(int(n)) for n in rng.integers(5, 30, size=9)], N=1, D=20,
                         H=128, C=999, rng=rng, inputs="all", labels="all")
    table = torch.from_numpy(rng.standard_normal((50, wl.D)).astype(np.float32)).cuda()
    words = rng.integers(-1, 50, wl.n_x).astype(np.int32)
    ctx = B.Context(0)
    want = LmBatch(wl, table, words, ctx, head_dtype=head_dtype).run()
    torch.cuda.synchronize()
    own = B.Context(0, torch.cuda.Stream())
    b = LmBatch(wl, table, words, own, head_dtype=head_dtype)
    b.schedule()
    b.alloc()
    kept = []
    for k in range(20):
        b.forward()
        kept.append(torch.full((1,), float(k + 1), device="cuda"))
        b.backward()
        b.infer()
        kept.append(torch.full((1,), float(k + 1), device="cuda"))
    own.sync()
    torch.cuda.synchronize()
    assert [float(t) for t in kept] == [k + 1.0 for k in range(20) for _ in range(2)]
    got = b.results()
    for k in want:
        assert np.array_equal(got[k], want[k]), k
    own.close()
    ctx.close()
