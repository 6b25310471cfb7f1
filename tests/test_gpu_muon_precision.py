"""How near the Newton-Schulz results are to the fp32 and fp64 ones where the
other tests' bounds are wide, in every form that a call can take.  bf16
matrices go through the steps of fp32 ones: their results are the fp32 results
of the same values, rounded once, bit for bit.
"""
import numpy as np
import pytest
import torch

from paper_2404_11068_amd import optim as op

pytestmark = pytest.mark.gpu

# matrices, rows, columns: in LDS; a workgroup each, of up to 128 rows and of up to 256; tiles of 64 x 64; of 128 x 128
FORMS = [(1, 64, 64), (2, 352, 96), (3, 33, 7), (75, 100, 700), (73, 250, 161), (72, 256, 256), (1, 300, 260), (5, 200, 640),
         (1, 1930, 2010), (45, 300, 260)]
IDS = lambda f: "%dx%dx%d" % f


BF16 = FORMS + [(2, 128, 224), (2, 576, 64), (2, 1216, 32), (78, 130, 200), (80, 520, 120), (1, 150, 280), (24, 700, 390), (1, 1, 7)]


@pytest.mark.parametrize("form", BF16, ids=IDS)
def test_bf16_is_the_fp32_result_rounded(form):
    print("\n[case] bf16", form, flush=True)
    N, m, n = form
    rng = np.random.default_rng(1)
    kinds = [rng.standard_normal((N, m, n)), np.einsum("km,kn->kmn", *(rng.standard_normal((N, s)) for s in (m, n)))]
    kinds.append(kinds[0] * np.exp(-9 * rng.random((N, m, 1))) * 1e-20)
    for x in kinds:
        t = torch.from_numpy(x).to(torch.bfloat16).cuda()
        for steps in (1, 2, 3, 5, 8):
            got, full = (op.orthogonalize(v, steps=steps, eps=1e-30) for v in (t, t.float()))
            assert full.any() and torch.equal(got, full.to(torch.bfloat16)), steps
