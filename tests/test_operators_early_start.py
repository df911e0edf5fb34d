"""Kernels that start while the one before them on the stream still runs read what that one writes.

On the CPU: their sources use no load of data taken for constant (its result is undefined where the data changes while a kernel lives).
On the GPU: calls whose inputs are the outputs of the call just before, with nothing between the two launches."""
import os
import re

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2102_06280_b200", "csrc")


@pytest.mark.parametrize("name", ["rows.cuh", "row_loss.cu", "lowrank.cu"])
def test_no_constant_cache_loads(name):
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert not re.findall(r"__ldg|__restrict__|ld\.global\.nc|ldu\.global", code)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,rows", [(300, 5000), (3000, 1500), (20000, 400), (70000, 300)])
def test_each_call_reads_what_the_one_before_wrote(vocab, rows):
    """The log-probabilities of one pass are the old ones of the next, its row losses the advantages, and then the weights, of later ones."""
    torch = pytest.importorskip("torch")
    import paper_2102_06280_b200 as p
    h = p.Dbw(np.array([0, 1, 2], np.int32), np.array([1, 0], np.int32), d=4)
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = (3 * torch.randn(rows, vocab, device="cuda", generator=gen)).bfloat16()
    action = torch.randint(0, vocab, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    rowstart = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")

    def chain(wait):
        old, adv, weight = torch.full((rows,), -9.0, device="cuda"), torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda")
        out = [[torch.zeros(rows, device="cuda") for _ in range(8)] for _ in range(2)]
        torch.cuda.synchronize()
        for k in range(8):
            h.policy_loss(z, action, old, adv, rowstart, out[0][k], logp=out[1][k], temperature=1.0 + 0.02 * k, row_weight=weight)
            old = out[1][k]
            adv, weight = (out[0][k], weight) if k % 2 else (adv, out[0][k])
            if wait:
                torch.cuda.synchronize()
        return out

    want = chain(True)
    for _ in range(5):
        for a, b in zip(sum(want, []), sum(chain(False), [])):
            assert torch.equal(a, b)
    assert h.status() == 0
