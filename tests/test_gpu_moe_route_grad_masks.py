"""tl_moe_route_grad: every number of lanes and of logits a lane, masked choices whose gradient is not finite, logits that are not numbers."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import moe_train as o
from tests.moe_train_util import Lib, choose, within
from tests.test_gpu_moe_route_grad import bound, grad

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")

# kernel (lanes of a token, logits of a lane), tokens, experts, choices
SHAPES = [("16 1", 33, 9, 3), ("16 2", 40, 32, 5), ("16 4", 65, 33, 8), ("16 8", 20, 128, 16), ("16 16", 50, 200, 7), ("32 1", 9, 32, 17), ("32 2", 70, 50, 20),
          ("32 4", 41, 100, 32), ("32 8", 37, 200, 17)]


def normal(T, E, k):
    rng = np.random.default_rng(T + E + k)
    f32 = lambda *s: rng.normal(size=s).astype(np.float32).astype(np.float64)
    return f32(T, E) * 2, choose(rng, T, E, k), f32(T, k)


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("kernel,T,E,k", SHAPES, ids=str)
def test_gradient(kernel, T, E, k, renormalize):
    logits, ids, dw = normal(T, E, k)
    within(grad(logits, ids, dw, renormalize), o.route_grad(logits, ids, dw, renormalize), bound(logits, ids, dw, renormalize), "dlogits")


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("kernel,T,E,k", SHAPES, ids=str)
def test_what_a_masked_choice_is_given_does_not_count(kernel, T, E, k, renormalize):
    """Logits of -inf, chosen: no weight and no gradient, whatever their dtopk_w."""
    logits, ids, dw = normal(T, E, k)
    given = dw.copy()
    for t in range(T):
        for j, bad in zip(range(t % 3 % k), (NAN, INF)):         # none, one or two of the choices
            logits[t, ids[t, j]] = -np.inf
            dw[t, j], given[t, j] = 0, bad if t % 2 else -bad
    got = grad(logits, ids, given, renormalize)
    within(got, o.route_grad(logits, ids, dw, renormalize), bound(logits, ids, dw, renormalize), "dlogits")
    assert not got[~np.isfinite(logits)].any()


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("kernel,T,E,k", SHAPES, ids=str)
def test_logits_that_are_not_numbers_are_not_masks(kernel, T, E, k, renormalize):
    """A token with such a logit, alone, among finite ones or beside masked ones, has no weights that are numbers: so are the gradients of all
    its logits, of the chosen ones with renormalize, but those of -inf.  The other tokens are as they would be."""
    logits, ids, dw = normal(T, E, k)
    clean = o.route_grad(logits, ids, dw, renormalize)
    size = bound(logits, ids, dw, renormalize)
    first = ids[:, 0]
    logits[0] = NAN
    logits[1, first[1]] = NAN
    logits[2] = -np.inf
    logits[2, first[2]] = NAN
    got = grad(logits, ids, dw, renormalize)
    for t in range(3):
        hit = np.zeros(E, bool)
        hit[ids[t] if renormalize else slice(None)] = True
        hit &= logits[t] != -np.inf
        assert np.isnan(got[t, hit]).all() and not got[t, ~hit].any(), t
    within(got[3:], clean[3:], size[3:], "dlogits")


def test_logits_beyond_32_bits():
    """2^24 tokens of 256 experts, 16 GiB, in place: equal logits, so that every weight is 2^-8 and all results are exact."""
    T, E = 1 << 24, 256
    logits, ids, dw = torch.zeros(T, E, device="cuda"), torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.zeros(T, 1, device="cuda")
    tokens = [0, 1 << 22, (1 << 23) + 1, T - 1]
    chosen = torch.tensor([255, 3, 0, 129], device="cuda")
    ids[tokens, 0], dw[tokens, 0] = chosen.int(), 65536.0
    with Lib() as ctx:
        tl.tl_moe_route_grad(ctx, logits, ids, dw, T, E, 1, 0, logits)
        ref = torch.full((len(tokens), E), -1.0, device="cuda")
        ref[torch.arange(len(tokens)), chosen] = 255.0
        assert torch.equal(logits[tokens], ref)
        logits[tokens] = 0
        assert not logits.any().item()
