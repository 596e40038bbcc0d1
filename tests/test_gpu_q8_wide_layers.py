"""Products of one to eight tokens with layers so wide that a block takes 32 rows: projections into a gated block, vocabularies."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from test_gpu_q8_linear import activations, kept, on_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nm():
    from paper_2507_17301_b200 import nm as mod
    return mod


def wide_layer(c_out, k, n, m, tile, seed):
    """(values, scales, indices, dense float64) of a random layer, on the GPU."""
    g = torch.Generator().manual_seed(seed)
    n_tiles, kk = -(-c_out // tile), kept(k, n, m)
    order = torch.rand((n_tiles, -(-k // m) * m), generator=g)
    order[:, k:] = 2.0
    keep = (order.view(n_tiles, -1, m).argsort(-1).argsort(-1) < n).view(n_tiles, -1)[:, :k]
    indices = keep.nonzero()[:, 1].view(n_tiles, kk)
    values = torch.randint(-127, 128, (c_out, kk), generator=g).to(torch.int8)
    values[0] = 127
    dense = torch.zeros(c_out, k, dtype=torch.float64).scatter_(1, indices.repeat_interleave(tile, 0)[:c_out], values.double())
    scales = torch.exp(torch.randn(c_out, generator=g)) / 5000
    return values.cuda(), scales.cuda(), indices.to(torch.uint16).cuda(), dense.cuda()


def close(y, x, xs, dense, ws, bias):
    u = 2.0 ** -24
    prod = (torch.from_numpy(x).cuda().double() @ dense.T) * torch.from_numpy(xs).cuda().double()[:, None] * ws.double()
    want = prod if bias is None else prod + bias.double()
    limit = prod.abs() * 2 * u * (1 + 4 * u) + want.abs() * u
    half = ref.STEP[y.dtype] if y.dtype != torch.float32 else 0.0
    limit = limit + (want.abs() + limit) * half + (2.0 ** -25 if y.dtype == torch.float16 else 2.0 ** -126)
    assert want.abs().max() < 65000
    assert torch.all((y.double() - want).abs() <= limit), ((y.double() - want).abs() / limit).max()


# tiles of 2 to 32 groups of eight rows, whole and not; rows that end inside a tile, a group, a block; columns that end inside a chunk
@pytest.mark.parametrize("c_out,k,n,m,tile", [
    (4800, 256, 2, 4, 64), (4737, 333, 2, 4, 64), (12288, 513, 2, 4, 64), (6000, 1000, 1, 4, 32), (3801, 130, 3, 4, 25), (5003, 700, 2, 8, 256),
    (9001, 77, 4, 8, 100), (5121, 64, 1, 8, 40), (20011, 300, 2, 4, 128), (7777, 515, 1, 1, 64), (4745, 128, 4, 4, 3), (16384, 65, 7, 11, 72)])
def test_one_to_eight_tokens(nm, c_out, k, n, m, tile):
    v, s, i, dense = wide_layer(c_out, k, n, m, tile, seed=c_out)
    h = nm.nm_q8_weights_import(v, s, i, k, n, m, tile)
    x, xs = activations(8, k)
    xg, xsg = on_gpu(x), torch.from_numpy(xs).cuda()
    bias = torch.randn(c_out, generator=torch.Generator().manual_seed(1)).cuda()
    for tokens in range(1, 9):
        for dtype, b in ((torch.float32, None), (torch.bfloat16, bias), (torch.float16, bias)):
            buf = torch.full((tokens + 2, c_out + 5), 3.0, dtype=dtype, device="cuda")
            y = nm.nm_q8_linear(h, xg[-tokens:], xsg[-tokens:], bias=b, y=buf[1:-1, 2:c_out + 2])
            close(y, x[-tokens:], xs[-tokens:], dense, s, b)
            buf[1:-1, 2:c_out + 2] = 3.0
            assert torch.all(buf == 3.0)
    nm.nm_q8_weights_check(h)


@pytest.mark.parametrize("n,m", [(2, 4), (1, 1)])
def test_sums_beyond_exact_32_bit_floats(nm, n, m):
    """More columns for a warp than fp32 adds up exactly at a time, and the least integers."""
    k, c_out, tile = 20000, 4800, 64
    v, s, i, dense = wide_layer(c_out, k, n, m, tile, seed=3)
    cols = i.long().repeat_interleave(tile, 0)[:c_out]
    x, xs = np.full((8, k), 127, dtype=np.int8), np.full(8, 1e-3, dtype=np.float32)
    x[:, 1::7] = 125
    x[3] = -128
    for least in (False, True):
        v[:] = -128 if least else torch.where(torch.rand(v.shape, device="cuda") < 0.5, 127, 126).to(torch.int8)
        dense.zero_().scatter_(1, cols, v.double())
        h = nm.nm_q8_weights_import(v, s / 100, i, k, n, m, tile)
        for tokens in (1, 2, 4, 5, 8):
            y = nm.nm_q8_linear(h, on_gpu(x[:tokens]), torch.from_numpy(xs[:tokens]).cuda(), out_dtype=torch.float32)
            close(y, x[:tokens], xs[:tokens], dense, s / 100, None)


def test_a_token_is_the_same_in_any_batch(nm):
    v, s, i, _ = wide_layer(9000, 1024, 2, 4, 64, seed=4)
    h = nm.nm_q8_weights_import(v, s, i, 1024, 2, 4, 64)
    x, xs = activations(300, 1024)
    xg, xsg = on_gpu(x), torch.from_numpy(xs).cuda()
    whole = nm.nm_q8_linear(h, xg, xsg, out_dtype=torch.float32)
    for tokens in (1, 2, 3, 4, 5, 7, 8, 9, 40):
        assert torch.equal(nm.nm_q8_linear(h, xg[:tokens], xsg[:tokens], out_dtype=torch.float32), whole[:tokens]), tokens


@pytest.mark.parametrize("tokens", [1, 8])
def test_a_token_that_is_not_finite_stays_alone(nm, tokens):
    v, s, i, _ = wide_layer(5000, 256, 2, 4, 64, seed=5)
    h = nm.nm_q8_weights_import(v, s, i, 256, 2, 4, 64)
    x, xs = activations(tokens, 256)
    xs[tokens // 2] = np.nan
    y = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda())
    assert torch.isnan(y[tokens // 2]).all() and int(torch.isnan(y).any(1).sum()) == 1
