"""What an 8-bit layer's handle keeps: the forms that a product reads, no more, and enough to export the layer again."""
import pytest
import torch

from test_gpu_q8_linear import kept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nm():
    from paper_2507_17301_b200 import nm as mod
    return mod


# bytes a dense weight: retained weights (n / m), 5/8 for the form of two of four columns or 1 for the expanded one, 2 n / m / tile for indices
@pytest.mark.parametrize("n,m,most", [(2, 4, 0.5 + 0.625 + 0.04), (1, 4, 0.25 + 0.625 + 0.02), (1, 8, 0.125 + 0.625 + 0.01), (3, 4, 0.75 + 1 + 0.04), (1, 1, 2.05)])
def test_device_memory_of_a_handle(nm, n, m, most):
    c_out, k, tile = 8192, 8192, 64
    w = torch.randn(c_out, k, device="cuda")
    nm.nm_q8_prune(w[:8, :64].contiguous(), n, m, 8).free()          # (what the first launch of a kernel loads)
    nm.nm_memory_trim()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    h = nm.nm_q8_prune(w, n, m, tile)
    nm.nm_memory_trim()
    used = free - torch.cuda.mem_get_info()[0]
    assert used <= most * c_out * k + (4 << 20), used / (c_out * k)
    h.free()
    nm.nm_memory_trim()
    assert torch.cuda.mem_get_info()[0] >= free - (2 << 20)


@pytest.mark.parametrize("c_out,k,n,m,tile", [(300, 1000, 2, 4, 64), (129, 257, 1, 4, 16), (70, 31, 2, 8, 8), (513, 640, 1, 2, 256), (40, 515, 3, 8, 1), (64, 3, 2, 4, 64),
                                              (130, 700, 3, 4, 32), (33, 130, 4, 8, 8), (260, 300, 1, 1, 64)])
def test_export_gives_back_what_was_imported(nm, c_out, k, n, m, tile):
    """Zeros among the retained weights, -128, and columns that stand together in some tiles."""
    g = torch.Generator().manual_seed(c_out)
    n_tiles, kk = -(-c_out // tile), kept(k, n, m)
    order = torch.rand((n_tiles, -(-k // m) * m), generator=g)
    order[::3] = order[::3].view(-1, -(-k // m), m).sort(-1).values.view(order[::3].shape)
    order[:, k:] = 2.0
    keep = (order.view(n_tiles, -1, m).argsort(-1).argsort(-1) < n).view(n_tiles, -1)[:, :k]
    indices = keep.nonzero()[:, 1].view(n_tiles, kk).to(torch.uint16)
    values = torch.randint(-128, 128, (c_out, kk), generator=g).to(torch.int8)
    values[torch.rand(values.shape, generator=g) < 0.3] = 0
    values[c_out // 2] = 0
    scales = torch.rand(c_out, generator=g)
    h = nm.nm_q8_weights_import(values.cuda(), scales.cuda(), indices.cuda(), k, n, m, tile)
    v, s, i = nm.nm_q8_weights_export(h)
    assert torch.equal(v.cpu(), values) and torch.equal(s.cpu(), scales) and torch.equal(i.cpu().int(), indices.int())
