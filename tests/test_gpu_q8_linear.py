"""nm_q8_prune, the handle, and nm_q8_linear against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import q8_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nm():
    from paper_2507_17301_b200 import nm as mod
    return mod


def kept(k, n, m):
    return k // m * n + min(k % m, n)


def layer(c_out, k, n, m, tile, seed=0):
    """(values, scales, indices) of a random layer."""
    rng = np.random.default_rng(seed)
    n_tiles = -(-c_out // tile)
    indices = np.empty((n_tiles, kept(k, n, m)), dtype=np.uint16)
    for t in range(n_tiles):
        cols = []
        for g in range(0, k, m):
            w = min(m, k - g)
            cols.extend(sorted(g + rng.choice(w, min(n, w), replace=False)))
        indices[t] = cols
    values = rng.integers(-127, 128, (c_out, indices.shape[1])).astype(np.int8)
    values[0, :] = -127 if seed % 2 else 127          # largest sums
    return values, np.exp(rng.normal(size=c_out)).astype(np.float32) / 500, indices


def activations(tokens, k, seed=0):
    rng = np.random.default_rng(seed + 100)
    x = rng.integers(-127, 128, (tokens, k)).astype(np.int8)
    x[-1] = 127
    return x, np.exp(rng.normal(size=tokens)).astype(np.float32) / 100


def on_gpu(x):
    """int8 rows as the quantising operators lay them out."""
    tokens, k = x.shape
    out = torch.empty_strided((tokens, k), ((k + 15) // 16 * 16, 1), dtype=torch.int8, device="cuda")
    out.copy_(torch.from_numpy(x))
    return out


def check(y, x, xs, dense, ws, bias, dtype):
    want, limit = ref.linear_limits(x, xs, dense, ws, bias, dtype)
    got = y.float().cpu().numpy().astype(np.float64)
    # sums beyond the type's range are infinities (65535 products of 127 * 127 times 0.0547 * 0.0097 are 5.6e5, fp16 ends at 65520)
    held = torch.from_numpy(want).to(dtype).double().numpy()
    over = np.isinf(held)
    assert np.array_equal(got[over], held[over])
    off = np.abs(np.where(over, 0.0, got - np.where(over, 0.0, want)))
    assert y.dtype == dtype and np.all(off <= limit), (np.max(off / limit), np.unravel_index(np.argmax(off / limit), off.shape))


def import_layer(nm, v, s, i, k, n, m, tile):
    return nm.nm_q8_weights_import(torch.from_numpy(v).cuda(), torch.from_numpy(s).cuda(), torch.from_numpy(i).cuda(), k, n, m, tile)


LAYERS = [  # c_out, k, n, m, tile
    (1, 1, 1, 1, 1), (8, 16, 2, 4, 8), (7, 15, 2, 4, 3), (64, 64, 2, 4, 64), (128, 128, 1, 4, 32), (129, 127, 3, 4, 16), (127, 129, 2, 8, 8),
    (257, 1000, 2, 4, 64), (1001, 1000, 2, 8, 8), (300, 513, 4, 8, 100), (256, 2048, 2, 4, 128), (96, 4096, 1, 8, 32), (520, 640, 1, 1, 64),
    (200, 777, 777, 777, 256), (192, 1024, 512, 1024, 64), (70, 3000, 7, 11, 24), (33, 260, 1, 2, 1), (24, 16384, 2, 4, 8), (16, 65535, 1, 1, 16),
]
TOKENS = [1, 2, 3, 7, 8, 9, 16, 17, 31, 33, 64, 65, 100, 128, 129, 200, 256, 257, 300]


@pytest.mark.parametrize("c_out,k,n,m,tile", LAYERS)
def test_linear_against_64_bits(nm, c_out, k, n, m, tile):
    v, s, i = layer(c_out, k, n, m, tile, seed=c_out)
    h = import_layer(nm, v, s, i, k, n, m, tile)
    assert (h.c_out, h.k, h.kk, h.n_tiles, h.tile_t) == (c_out, k, v.shape[1], i.shape[0], tile)
    dense = ref.dense_of(v, i, k, tile)
    x, xs = activations(max(TOKENS), k)
    bias = np.random.default_rng(1).normal(size=c_out).astype(np.float32)
    xg, xsg, bg = on_gpu(x), torch.from_numpy(xs).cuda(), torch.from_numpy(bias).cuda()
    for at, tokens in enumerate(TOKENS):
        dtype = (torch.bfloat16, torch.float32, torch.float16)[at % 3]
        with_bias = at % 2 == 1
        y = nm.nm_q8_linear(h, xg[-tokens:], xsg[-tokens:], bias=bg if with_bias else None, out_dtype=dtype)
        nm.nm_q8_weights_check(h)
        check(y, x[-tokens:], xs[-tokens:], dense, s, bias if with_bias else None, dtype)


def test_a_token_is_the_same_in_any_batch(nm):
    """Sums are exact, so the result does not depend on the kernel, the split or the other tokens."""
    v, s, i = layer(384, 2048, 2, 4, 64)
    h = import_layer(nm, v, s, i, 2048, 2, 4, 64)
    x, xs = activations(700, 2048)
    xg, xsg = on_gpu(x), torch.from_numpy(xs).cuda()
    whole = nm.nm_q8_linear(h, xg, xsg, out_dtype=torch.float32)
    for tokens in (1, 5, 8, 12, 30, 60, 128, 250, 600):
        assert torch.equal(nm.nm_q8_linear(h, xg[:tokens], xsg[:tokens], out_dtype=torch.float32), whole[:tokens]), tokens


@pytest.mark.parametrize("c_out,k,n,m,tile,tokens", [(4096, 4096, 2, 4, 64, 2000), (2000, 5000, 1, 4, 32, 515), (1280, 1536, 4, 4, 64, 4100)])
def test_large_products(nm, c_out, k, n, m, tile, tokens):
    """Against the exact sums of 64-bit floating point on the GPU (integers below 2^53)."""
    v, s, i = layer(c_out, k, n, m, tile)
    h = import_layer(nm, v, s, i, k, n, m, tile)
    x, xs = activations(tokens, k)
    dense = ref.dense_of(v, i, k, tile)
    sums = (torch.from_numpy(x).cuda().double() @ torch.from_numpy(dense).cuda().T)
    y = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda(), out_dtype=torch.float32)
    nm.nm_q8_weights_check(h)
    prod = sums * torch.from_numpy(xs).cuda().double()[:, None] * torch.from_numpy(s).cuda().double()
    assert torch.all((y.double() - prod).abs() <= prod.abs() * 3.1 * 2.0 ** -24 + 2.0 ** -126)


@pytest.mark.parametrize("c_out,k,n,m,tile", [(64, 96, 2, 4, 8), (100, 130, 1, 4, 32), (33, 77, 3, 5, 16), (40, 600, 300, 600, 8), (50, 64, 4, 4, 64)])
def test_prune_selects_as_the_oracle_and_rounds_to_nearest(nm, c_out, k, n, m, tile):
    g = torch.Generator().manual_seed(c_out)
    w = torch.randn((c_out, k), generator=g) * torch.exp(torch.randn((c_out, 1), generator=g))
    w[3] = 0
    h = nm.nm_q8_prune(w.cuda(), n, m, tile)
    values, scales, indices = (t.cpu() for t in nm.nm_q8_weights_export(h))
    want_v, want_i = oracle.prune(w.numpy().reshape(c_out, 1, 1, k), n, m, tile)
    assert np.array_equal(indices.numpy(), want_i)
    want_q, a = ref.quantised(torch.from_numpy(want_v.reshape(c_out, -1)).double())
    assert torch.equal(values, want_q)
    assert torch.all((scales.double() - a / 127.0).abs() <= a / 127.0 * 2.0 ** -24)
    # and the layer it makes computes with them
    x, xs = activations(40, k)
    for tokens in (1, 6, 40):
        y = nm.nm_q8_linear(h, on_gpu(x[:tokens]), torch.from_numpy(xs[:tokens]).cuda(), out_dtype=torch.float32)
        check(y, x[:tokens], xs[:tokens], ref.dense_of(values, indices, k, tile), scales.numpy(), None, torch.float32)


def test_weights_that_are_not_finite(nm):
    w = torch.randn(16, 32)
    w[2, 5], w[9, 0] = float("nan"), float("inf")
    h = nm.nm_q8_prune(w.cuda(), 2, 4, 8)
    values, scales, _ = nm.nm_q8_weights_export(h)
    bad = torch.tensor([o in (2, 9) for o in range(16)])
    assert torch.equal(torch.isnan(scales.cpu()), bad) and not values.cpu()[bad].any()
    for tokens in (1, 20):
        y = nm.nm_q8_linear(h, torch.ones(tokens, 32, dtype=torch.int8, device="cuda"), torch.ones(tokens, device="cuda"))
        assert torch.equal(torch.isnan(y.cpu()).all(0), bad) and torch.equal(torch.isnan(y.cpu()).any(0), bad)


def test_export_and_import_are_inverse(nm):
    for c_out, k, n, m, tile in ((70, 300, 2, 4, 16), (5, 33, 1, 8, 2), (64, 64, 1, 1, 64)):
        v, s, i = layer(c_out, k, n, m, tile)
        h = import_layer(nm, v, s, i, k, n, m, tile)
        gv, gs, gi = nm.nm_q8_weights_export(h)
        assert np.array_equal(gv.cpu().numpy(), v) and np.array_equal(gs.cpu().numpy(), s) and np.array_equal(gi.cpu().numpy(), i)


def test_bad_index_rows_are_refused(nm):
    v, s, i = layer(16, 64, 2, 4, 8)
    for at, value in ((0, 1), (31, 64), (31, 65535), (4, 3), (3, 3)):
        bad = i.copy()
        bad[0] = np.sort(bad[0])
        bad[0, at] = value if at != 0 else bad[0, 1]
        if np.array_equal(bad, i):
            continue
        ok = all(bad[0, j] // 4 == j // 2 and (j == 0 or bad[0, j] > bad[0, j - 1]) for j in range(32)) and bad[0, 31] < 64
        if ok:
            import_layer(nm, v, s, bad, 64, 2, 4, 8)
            continue
        with pytest.raises(nm.NmError) as e:
            import_layer(nm, v, s, bad, 64, 2, 4, 8)
        assert e.value.status == nm.NM_ERR_INVALID_ARG
    with pytest.raises(TypeError):
        import_layer(nm, v[:, :30], s, i, 64, 2, 4, 8)


@pytest.mark.parametrize("tokens", [1, 5, 24, 90, 300])
def test_a_token_that_is_not_finite_stays_alone(nm, tokens):
    v, s, i = layer(200, 256, 2, 4, 8)
    h = import_layer(nm, v, s, i, 256, 2, 4, 8)
    x, xs = activations(tokens, 256)
    xs[tokens // 2] = np.nan
    y = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda()).cpu()
    want = torch.zeros(tokens, dtype=torch.bool)
    want[tokens // 2] = True
    assert torch.equal(torch.isnan(y).all(1), want) and torch.equal(torch.isnan(y).any(1), want)


@pytest.mark.parametrize("tokens", [1, 4, 13, 50, 150, 280])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_outputs_in_larger_buffers(nm, tokens, dtype):
    """Rows before, after and beside the output stay as they were; activations may have any pitch that is a multiple of 16."""
    v, s, i = layer(130, 200, 2, 4, 32)
    h = import_layer(nm, v, s, i, 200, 2, 4, 32)
    x, xs = activations(tokens, 200)
    wide = torch.full((tokens, 320), 99, dtype=torch.int8, device="cuda")
    wide[:, 32:232].copy_(torch.from_numpy(x))
    buf = torch.full((tokens + 2, 137), 3.0, dtype=dtype, device="cuda")
    y = nm.nm_q8_linear(h, wide[:, 32:232], torch.from_numpy(xs).cuda(), y=buf[1:-1, 3:133])
    check(y, x, xs, ref.dense_of(v, i, 200, 32), s, None, dtype)
    buf[1:-1, 3:133] = 3.0
    assert torch.all(buf == 3.0)


def test_refusals(nm):
    v, s, i = layer(64, 100, 2, 4, 32)
    h = import_layer(nm, v, s, i, 100, 2, 4, 32)
    x, xs = activations(4, 100)
    xg, sg = on_gpu(x), torch.from_numpy(xs).cuda()
    for bad in (lambda: nm.nm_q8_linear(h, xg[:, :99], sg), lambda: nm.nm_q8_linear(h, xg, sg[:3]), lambda: nm.nm_q8_linear(h, xg.float(), sg),
                lambda: nm.nm_q8_linear(h, xg, sg, out_dtype=torch.float64), lambda: nm.nm_q8_linear(h, xg, sg, bias=sg),
                lambda: nm.nm_q8_linear(h, xg, sg, y=torch.empty(4, 63, device="cuda")), lambda: nm.nm_q8_linear(h, xg, sg.double())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: nm.nm_q8_linear(h, xg.contiguous(), sg), lambda: nm.nm_q8_linear(h, torch.zeros(4, 128, dtype=torch.int8, device="cuda")[:, 8:108], sg)):
        with pytest.raises(nm.NmError) as e:
            bad()
        assert e.value.status == nm.NM_ERR_INVALID_ARG
    assert nm.nm_q8_linear(h, xg[:0], sg[:0]).shape == (0, 64)
    h.free()
    with pytest.raises(nm.NmError):
        nm.nm_q8_linear(h, xg, sg)


@pytest.mark.parametrize("tokens", [1, 6, 20, 100, 400])
def test_two_streams_and_two_graphs_share_a_handle(nm, tokens):
    v, s, i = layer(512, 1024, 2, 4, 64)
    h = import_layer(nm, v, s, i, 1024, 2, 4, 64)
    data = [activations(tokens, 1024, seed=j) for j in range(2)]
    xg, sg = [on_gpu(x) for x, _ in data], [torch.from_numpy(xs).cuda() for _, xs in data]
    want = [nm.nm_q8_linear(h, a, b, out_dtype=torch.float32) for a, b in zip(xg, sg)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for j in range(2):
            with torch.cuda.stream(streams[j]):
                got[j].append(nm.nm_q8_linear(h, xg[j], sg[j], out_dtype=torch.float32))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[j]) for j in range(2) for y in got[j])
    graphs, outs = [], []
    for j in range(2):
        y = torch.empty_like(want[j])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            nm.nm_q8_linear(h, xg[j], sg[j], y=y)
        graphs.append(g)
        outs.append(y)
    for _ in range(10):
        for j in range(2):
            outs[j].zero_()
            streams[j].wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(streams[j]):
                graphs[j].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[j], want[j]) for j in range(2))
    nm.nm_q8_weights_check(h)


@pytest.mark.parametrize("tokens", [1, 7, 48, 300])
def test_a_gated_block(nm, tokens):
    """The operators together, as a pruned model's block runs them: norm with residual, two products, gate, product, next norm,
    in one stream and as a captured graph; against the same steps in 64 bits on the same 8-bit operands."""
    h, inner = 256, 520
    g = torch.Generator().manual_seed(tokens)
    w_up, w_down = torch.randn((2 * inner, h), generator=g) / 16, torch.randn((h, inner), generator=g) / 23
    up, down = nm.nm_q8_prune(w_up.cuda(), 2, 4, 8), nm.nm_q8_prune(w_down.cuda(), 1, 4, 64)
    norm = (1 + 0.1 * torch.randn(h, generator=g)).bfloat16()
    x, r = torch.randn((tokens, h), generator=g).bfloat16(), torch.randn((tokens, h), generator=g).bfloat16()
    xg, rg, ng = x.cuda(), r.cuda(), norm.cuda()

    def block():
        q, s, res = nm.nm_q8_rmsnorm(xg, ng, 1e-6, residual=rg)
        gate_up = nm.nm_q8_linear(up, q, s)
        q2, s2 = nm.nm_q8_silu_mul(gate_up[:, :inner], gate_up[:, inner:])
        y = nm.nm_q8_linear(down, q2, s2)
        return (q, s, res, gate_up, q2, s2, y) + tuple(nm.nm_q8_rmsnorm(y, ng, 1e-6, residual=res))

    got = block()
    torch.cuda.synchronize()
    q, s, res, gate_up, q2, s2, y, q3, s3, res3 = (t.cpu() for t in got)
    for handle, xq, xs, out in ((up, q, s, gate_up), (down, q2, s2, y)):
        v, ws, i = (t.cpu() for t in nm.nm_q8_weights_export(handle))
        check(out, xq.numpy(), xs.numpy(), ref.dense_of(v, i, handle.k, handle.tile_t), ws.numpy(), None, torch.bfloat16)
        nm.nm_q8_weights_check(handle)
    want = ref.rmsnorm(x, norm, 1e-6, r)
    assert torch.equal(q, want[0]) and torch.equal(res, want[2])
    assert torch.equal(q2, ref.silu_mul(gate_up[:, :inner], gate_up[:, inner:])[0])
    want = ref.rmsnorm(y, norm, 1e-6, res)
    assert torch.equal(q3, want[0]) and torch.equal(res3, want[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = block()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a.cpu(), b.cpu()) for a, b in zip(again, got))


@pytest.mark.parametrize("c_out,k,n,m,tile,tokens", [
    (1001, 300, 2, 4, 64, 2431), (300, 129, 1, 8, 16, 6500), (1500, 513, 3, 4, 32, 1700), (130, 77, 1, 2, 8, 9601), (2304, 1024, 2, 8, 100, 1111),
    (640, 640, 1, 1, 64, 3900), (4864, 2050, 1, 3, 64, 449), (257, 1, 1, 1, 64, 8000), (2560, 260, 2, 4, 1, 1025), (1024, 512, 4, 8, 64, 2432)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_many_tokens(nm, c_out, k, n, m, tile, tokens, dtype):
    """More tiles than SMs: pairs of CTAs, with and without sparse operands (two of four columns at most), aligned and unaligned
    outputs, against sums of integers in 64-bit floating point."""
    v, s, i = layer(c_out, k, n, m, tile, seed=k)
    v[1::3, ::2] = 0                                   # retained weights that are zero
    h = import_layer(nm, v, s, i, k, n, m, tile)
    x, xs = activations(tokens, k)
    s = (s / 20).astype(np.float32)                    # (fp16's range)
    h = import_layer(nm, v, s, i, k, n, m, tile)
    bias = np.random.default_rng(2).normal(size=c_out).astype(np.float32)
    dense = torch.from_numpy(ref.dense_of(v, i, k, tile)).cuda()
    prod = (torch.from_numpy(x).cuda().double() @ dense.T) * torch.from_numpy(xs).cuda().double()[:, None] * torch.from_numpy(s).cuda().double()
    want = prod + torch.from_numpy(bias).cuda().double()
    u = 2.0 ** -24
    limit = prod.abs() * 2 * u * (1 + 4 * u) + want.abs() * u
    half = ref.STEP[dtype] if dtype != torch.float32 else 0.0
    limit = limit + (want.abs() + limit) * half + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126)
    assert want.abs().max() < 65000
    wide = torch.full((tokens + 1, c_out + 3), 7.0, dtype=dtype, device="cuda")
    for out in (None, wide[:tokens, 1:c_out + 1]):
        y = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda(), bias=torch.from_numpy(bias).cuda(), out_dtype=dtype, y=out)
        nm.nm_q8_weights_check(h)
        assert torch.all((y.double() - want).abs() <= limit), ((y.double() - want).abs() / limit).max()
    wide[:tokens, 1:c_out + 1] = 7.0
    assert torch.all(wide == 7.0)


@pytest.mark.parametrize("tokens", [1, 2, 4, 8, 15, 70, 1400])
@pytest.mark.parametrize("n,m", [(2, 4), (1, 1)])
def test_the_least_integers(nm, tokens, n, m):
    """-128 on both sides, which the quantising operators never make but a checkpoint may hold: sums of 2^14 a column."""
    k, c_out = 2050, 1560
    _, s, i = layer(c_out, k, n, m, 40)
    v = np.full((c_out, i.shape[1]), -128, dtype=np.int8)
    h = import_layer(nm, v, s, i, k, n, m, 40)
    x = np.full((tokens, k), -128, dtype=np.int8)
    x[tokens // 2, ::3] = 127
    xs = np.ones(tokens, dtype=np.float32)
    y = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda(), out_dtype=torch.float32)
    check(y, x, xs, ref.dense_of(v, i, k, 40), s, None, torch.float32)


def test_more_sums_than_32_bit_floats_hold(nm):
    """Eight tokens of a long layer: a warp's part of the columns is more than fp32 adds up exactly at a time."""
    k, c_out = 40000, 64
    v, s, i = layer(c_out, k, 2, 4, 32)
    v[:] = np.where(np.random.default_rng(5).random(v.shape) < 0.5, 127, 126).astype(np.int8)
    h = import_layer(nm, v, s, i, k, 2, 4, 32)
    x = np.full((8, k), 127, dtype=np.int8)
    x[:, 1::7] = 125
    xs = np.ones(8, dtype=np.float32)
    for tokens in (1, 2, 3, 5, 8):
        y = nm.nm_q8_linear(h, on_gpu(x[:tokens]), torch.from_numpy(xs[:tokens]).cuda(), out_dtype=torch.float32)
        check(y, x[:tokens], xs[:tokens], ref.dense_of(v, i, k, 32), s, None, torch.float32)


def test_pruning_rules_of_four_columns(nm):
    """Sparse operands need at most two retained columns of four aligned ones, whatever the weights: patterns on either side of
    that, and wherever the columns lie."""
    for n, m in ((1, 2), (1, 3), (2, 5), (2, 6), (2, 7), (2, 8), (3, 8), (3, 12), (1, 6), (5, 16)):
        k, c_out, tokens = 333, 200, 40
        v, s, i = layer(c_out, k, n, m, 16, seed=n * m)
        for t in range(i.shape[0]):                                    # columns pushed together at one end of each group
            if t % 3:
                i[t] = [g + (c if t % 3 == 1 else min(m, k - g) - min(n, k - g) + c) for g in range(0, k, m) for c in range(min(n, k - g))]
        h = import_layer(nm, v, s, i, k, n, m, 16)
        x, xs = activations(tokens, k)
        y = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda(), out_dtype=torch.float32)
        check(y, x, xs, ref.dense_of(v, i, k, 16), s, None, torch.float32)


@pytest.mark.parametrize("tokens,x_ld,y_ld,c_out", [(3, 2 ** 31 + 64, 2 ** 30 + 4, 130), (40, 2 ** 27, 2 ** 26 + 1, 130), (1100, 2 ** 22 + 16, 2 ** 21 + 4, 2200)])
def test_offsets_past_32_bits(nm, tokens, x_ld, y_ld, c_out):
    """Rows of activations and outputs gigabytes apart, in each kernel, and rows of the operators that make them."""
    k = 520
    v, s, i = layer(c_out, k, 2, 4, 32)
    h = import_layer(nm, v, s, i, k, 2, 4, 32)
    x, xs = activations(tokens, k)
    xb = torch.zeros((tokens - 1) * x_ld + 1024, dtype=torch.int8, device="cuda")
    yb = torch.zeros((tokens - 1) * y_ld + 4096, dtype=torch.float32, device="cuda")
    xg, y = xb.as_strided((tokens, k), (x_ld, 1)), yb.as_strided((tokens, c_out), (y_ld, 1))
    xg.copy_(torch.from_numpy(x))
    nm.nm_q8_linear(h, xg, torch.from_numpy(xs).cuda(), y=y)
    nm.nm_q8_weights_check(h)
    check(y, x, xs, ref.dense_of(v, i, k, 32), s, None, torch.float32)
    a = yb.as_strided((tokens, k), (y_ld, 1))
    a.copy_(torch.randn(tokens, k, generator=torch.Generator().manual_seed(3)))
    q, scale = nm.nm_q8_rows(a, q=xg)
    assert q.data_ptr() == xg.data_ptr() and torch.equal(q.cpu(), ref.rows(a.cpu())[0])
    w = torch.randn(k, generator=torch.Generator().manual_seed(4))
    want_q, _, want_r = ref.rmsnorm(a.cpu(), w, 1e-6, a.cpu())
    q, scale, r = nm.nm_q8_rmsnorm(a, w.cuda(), 1e-6, residual=a, residual_out=a, q=xg)
    assert torch.equal(r.cpu(), want_r) and torch.equal(q.cpu(), want_q)


@pytest.mark.parametrize("c_out,tokens", [(4096, 9), (4096, 100), (4096, 333), (4096, 512), (12288, 20), (12288, 61), (12288, 128), (20000, 11), (20000, 77), (20000, 128),
                                          (1100, 640), (700, 30), (2200, 40)])
@pytest.mark.parametrize("k,n,m", [(700, 2, 4), (1300, 4, 4)])
def test_middling_tokens(nm, c_out, tokens, k, n, m):
    """Tiles of 16 to 128 tokens, split and whole, one round of them and more, sparse and dense."""
    v, s, i = layer(c_out, k, n, m, 64, seed=3)
    h = import_layer(nm, v, s, i, k, n, m, 64)
    x, xs = activations(tokens, k)
    dense = torch.from_numpy(ref.dense_of(v, i, k, 64)).cuda()
    prod = (torch.from_numpy(x).cuda().double() @ dense.T) * torch.from_numpy(xs).cuda().double()[:, None] * torch.from_numpy(s).cuda().double()
    buf = torch.full((tokens + 1, c_out), 5.0, device="cuda")
    y = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda(), y=buf[:tokens])
    nm.nm_q8_weights_check(h)
    assert torch.all((y.double() - prod).abs() <= prod.abs() * 3.1 * 2.0 ** -24 + 2.0 ** -126)
    assert torch.all(buf[tokens] == 5.0)
    half = nm.nm_q8_linear(h, on_gpu(x), torch.from_numpy(xs).cuda(), out_dtype=torch.bfloat16)
    assert torch.all((half.double() - prod).abs() <= prod.abs() * (2.0 ** -8 + 2.0 ** -20) + 2.0 ** -126)


@pytest.mark.parametrize("n,m", [(2, 2 ** 31 - 1), (24, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1), (2, 2 ** 30 + 1)])
def test_groups_longer_than_a_row(nm, n, m):
    # one group, of the k columns that exist
    k, c_out = 100, 48
    w = torch.randn(c_out, k, generator=torch.Generator().manual_seed(5)).cuda()
    far, near = nm.nm_q8_prune(w, n, m, 16), nm.nm_q8_prune(w, min(n, k), k, 16)
    v, s, i = nm.nm_q8_weights_export(far)
    for got, want in zip((v, s, i), nm.nm_q8_weights_export(near)):
        assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
    again = nm.nm_q8_weights_import(v, s, i, k, n, m, 16)
    for tokens in (1, 20):
        x, xs = nm.nm_q8_rows(torch.randn(tokens, k, generator=torch.Generator().manual_seed(tokens)).cuda())
        want = nm.nm_q8_linear(near, x, xs, out_dtype=torch.float32)
        assert torch.equal(nm.nm_q8_linear(far, x, xs, out_dtype=torch.float32), want)
        assert torch.equal(nm.nm_q8_linear(again, x, xs, out_dtype=torch.float32), want)
