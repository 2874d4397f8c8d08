"""The operators around drafting on the GPU: numbers at the ends of their ranges."""
import math

import numpy as np
import pytest
import torch

import paper_2502_20704_amd as fsd
from tests.test_drafting_gpu import DT, _dev, _host

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ normalisers


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,times", [(50, 1), (9002, 1), (100002, 10)])   # (30 long rows a number: by the kernel with the table)
def test_select_rows_of_one_large_number(V, times, dtype):
    """A row is as likely as it is a number higher up or lower down, however large that number is: where a mask of the type's lowest number leaves a beam
    nothing, each of its V entries has the score -log V, and does not stand in front of beams that have something."""
    numbers = [torch.finfo(DT[dtype]).min, -1e30, 2.0 ** 100, -(2.0 ** 60)] * times
    B, n = len(numbers), 8
    z = torch.empty((B, 3, V), dtype=DT[dtype])
    z[:, 0] = torch.tensor(numbers, dtype=DT[dtype])[:, None]
    z[:, 1], z[:, 1, 5:8] = -math.inf, 0.25
    z[:, 2], z[:, 2, ::2] = -math.inf, torch.tensor(numbers, dtype=DT[dtype])[:, None]
    scores = np.array([[-1.0, -1.5, -1.75]] * B, np.float32)
    got = fsd.fsd_beam_select(z.cuda(), _dev(scores), n)
    torch.cuda.synchronize()
    assert not got["row_status"].any()
    # -1.5 - log 3; then -1.75 - log V + log 2 = -1.057 - log V is behind -1 - log V
    assert (_host(got["parent"]) == [1, 1, 1, 0, 0, 0, 0, 0]).all() and (_host(got["tokens"]) == [5, 6, 7, 0, 1, 2, 3, 4]).all()
    want = np.array([-1.5 - math.log(3)] * 3 + [-1.0 - math.log(V)] * 5)
    # one rounding to binary32, and the normaliser's error
    assert (np.abs(_host(got["scores"]) - want) <= 2.0 ** -24 * np.abs(want) * (1 + 2.0 ** -20) + 2.0 ** -32).all()


def test_select_normaliser_within_its_bound():
    """The sum of a row's exponentials is off by less than 2^-33 of it, also where every entry's exponential is formed from a wavefront's largest entry, that
    from the slice's and that from the row's, each at a distance at which the polynomial is off the most.  (Rows beyond the range of e^z; parts of
    256 entries are the wavefronts' of a call of this size.)"""
    V, far = 65536, 218 * 2.0 ** -14                          # a multiple of the numbers' distance there
    z = np.full((V // 1024, 4, 256), 1000.0 - 3 * far)
    z[:, :, 0] += far                                         # a part's largest
    z[:, 0] = -np.inf
    z[:, 0, 0] = 1000.0 - far                                 # a slice's, alone in its part
    z[0, 0, 0] = 1000.0                                       # the row's
    z = z.reshape(1, 1, V).astype(np.float32)
    least = z[0, 0].astype(np.float64) - 1000.0
    norm = math.log(math.fsum(np.exp(least[least > -np.inf]).tolist()))
    scores = np.array([[norm]], np.float32)                   # (so that the result is near 0, and its rounding small)
    got = fsd.fsd_beam_select(_dev(z), _dev(scores), 1)
    want = float(scores[0, 0]) - norm
    assert int(got["tokens"][0, 0]) == 0
    assert abs(float(got["scores"][0, 0]) - want) <= 2.0 ** -33 + 2.0 ** -24 * abs(want) + 2.0 ** -45


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,B", [(40, 4), (9000, 4), (100003, 14)])
def test_select_only_continuations_are_certain(V, B, dtype):
    """A row with one entry gives the beam's score itself, so that it ties with a finished beam of that score and with other such rows: the lowest beam comes
    first, whatever the logits are."""
    rng = np.random.default_rng(V)
    W = 6
    z = torch.full((B, W, V), -math.inf, dtype=DT[dtype])
    at = rng.integers(0, V, (B, W))
    values = rng.standard_normal((B, W)) * 4
    values[1] = rng.standard_normal(W) * 300                  # beyond the table's range, and e^z's
    values[2] = rng.uniform(-1e30, 1e30, W)
    values[3, :3], values[3, 3:] = [0.0, 64.0, -63.5], [1e-30, -2.0 ** -13, 600.0]
    for b in range(B):
        for w in range(W):
            z[b, w, at[b, w]] = float(values[b, w])
    scores = np.full((B, W), -2.3, np.float32)
    done = np.zeros((B, W), np.int32)
    done[0, 2] = done[2, 3] = 1
    for n in (1, 4, 9):
        got = fsd.fsd_beam_select(z.cuda(), _dev(scores), n, done=_dev(done))
        k = min(n, W)
        assert not got["row_status"].any()
        assert (_host(got["parent"])[:, :k] == np.arange(k)).all() and (_host(got["parent"])[:, k:] == -1).all()
        assert (_host(got["tokens"])[:, :k] == np.where(done[:, :k] != 0, -1, at[:, :k])).all()
        assert (_host(got["scores"])[:, :k] == scores[:, :k]).all()
    # (0 is no size to measure an error of 2^-33 by: exactly 0)
    got = fsd.fsd_beam_select(z.cuda(), None, 4)
    assert (got["scores"] == 0.0).all() and (_host(got["parent"]) == np.arange(4)).all()
