"""A wait of the 8-bit product that expires: no output is written from the sums that are there by then, the status says so once, and
the handle goes on as before."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from test_gpu_q8_linear import activations, check, import_layer, layer, on_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nm():
    from paper_2507_17301_b200 import nm as mod
    return mod


# one round of tiles, more than one (two CTAs on an SM), sparse and dense weights, and a reduction axis shared by clusters of 2 and 4
# (blocks of 256 columns at 2:4, of 128 dense).  A wait that expires takes seconds, so there are few cases.
@pytest.mark.parametrize("c_out,k,n,m,tokens,block", [(300, 100, 2, 4, 70, 0), (20000, 3000, 2, 4, 77, 6), (20000, 2500, 1, 1, 128, 19),
                                                      (256, 2048, 2, 4, 20, 3), (3000, 2000, 1, 1, 40, 15)])
def test_nothing_is_written_from_unfinished_sums(nm, c_out, k, n, m, tokens, block):
    v, s, i = layer(c_out, k, n, m, 64)
    h = import_layer(nm, v, s, i, k, n, m, 64)
    x, xs = activations(tokens, k)
    xg, xsg = on_gpu(x), torch.from_numpy(xs).cuda()
    y = torch.full((tokens, c_out), 7.0, device="cuda")
    nm.nm_selftest_q8_wait_expiry(h, xg, xsg, y, block=block)
    with pytest.raises(nm.NmError) as e:
        nm.nm_q8_weights_check(h)
    assert e.value.status == nm.NM_ERR_TIMEOUT
    assert torch.all(y == 7.0)
    nm.nm_q8_weights_check(h)                                              # reported once
    nm.nm_selftest_q8_wait_expiry(h, xg, xsg, y, block=-(-k // 128))            # no such block: the product
    nm.nm_q8_weights_check(h)
    want = nm.nm_q8_linear(h, xg, xsg, out_dtype=torch.float32)
    nm.nm_q8_weights_check(h)
    assert torch.equal(y, want)
    if c_out < 1000:
        check(y, x, xs, ref.dense_of(v, i, k, 64), s, None, torch.float32)


def test_refusals(nm):
    v, s, i = layer(64, 100, 2, 4, 32)
    h = import_layer(nm, v, s, i, 100, 2, 4, 32)
    x, xs = activations(4, 100)
    xg, sg, y = on_gpu(x), torch.from_numpy(xs).cuda(), torch.zeros(4, 64, device="cuda")
    with pytest.raises(nm.NmError) as e:
        nm.nm_selftest_q8_wait_expiry(h, xg, sg, y, block=-1)
    assert e.value.status == nm.NM_ERR_INVALID_ARG
    for bad in ((xg[:3], sg, y), (xg, sg[:3], y), (xg, sg, y.half()), (xg.float(), sg, y)):
        with pytest.raises(TypeError):
            nm.nm_selftest_q8_wait_expiry(h, *bad)
    assert np.all(y.cpu().numpy() == 0)
