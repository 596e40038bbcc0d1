"""nm_q8_rmsnorm, nm_q8_silu_mul, nm_q8_rows against their definitions in 64 bits: the integers are equal, the scales within
their roundings."""
import pytest
import torch

import q8_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
# Scale of a norm: a sum of h squares in 32 bits, every term passes at most max(32, h / 512) + 10 roundings of 2^-24 (terms a thread
# adds up, then two trees), which the root halves; mean, eps, root, reciprocal, a / 127 and the last product: 6 more.
NORM_SCALE = 2.0 ** -24


@pytest.fixture(scope="module")
def nm():
    from paper_2507_17301_b200 import nm as mod
    return mod


def norm_limit(h):
    return ((max(32, h / 512 + 32) + 10) / 2 + 6) * NORM_SCALE


def randn(*shape, seed=0, dtype=torch.float32, spread=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if spread and len(shape) == 2:
        x = x * torch.exp(torch.randn((shape[0], 1), generator=g))
    return x.to(dtype)


def same_scale(got, want, limit):
    got = got.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert torch.all((got - want).abs()[fine] <= want[fine] * limit + 2.0 ** -149)


# widths around every limit of the kernels' shapes: a group of eight, 1024, 4096, 8192, 16384, and beyond; odd ones
WIDTHS = [1, 7, 8, 9, 31, 64, 100, 255, 1000, 1001, 1024, 1032, 2049, 4096, 4104, 5000, 8191, 8192, 8200, 16384, 16400, 20001, 32768, 65535]


@pytest.mark.parametrize("h", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [3, 299])
def test_rmsnorm_widths(nm, h, dtype, tokens):
    if tokens > 100 and h > 20001:
        tokens = 297
    x, r, w = randn(tokens, h, seed=1, dtype=dtype), randn(tokens, h, seed=2, dtype=dtype), randn(h, seed=3, dtype=dtype)
    x[1] = 0
    r[1] = 0
    want_q, want_s, want_r = ref.rmsnorm(x, w, 1e-5, r)
    q, s, out = nm.nm_q8_rmsnorm(x.cuda(), w.cuda(), 1e-5, residual=r.cuda())
    assert torch.equal(out.cpu(), want_r)
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, norm_limit(h))


@pytest.mark.parametrize("h", [8, 100, 1001, 4096, 8192, 20001])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [1, 300])
def test_rows_and_silu_mul_widths(nm, h, dtype, tokens):
    x, u = 3 * randn(tokens, h, seed=4, dtype=dtype), randn(tokens, h, seed=5, dtype=dtype)
    want_q, want_s = ref.rows(x)
    q, s = nm.nm_q8_rows(x.cuda())
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, 2.0 ** -24)
    want_q, want_s = ref.silu_mul(x, u)
    q, s = nm.nm_q8_silu_mul(x.cuda(), u.cuda())
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, 2.0 ** -24)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_fp32_norm_weights_beside_16_bit_activations(nm, dtype):
    x, w = randn(40, 1000, seed=6, dtype=dtype), randn(1000, seed=7)
    want_q, want_s = ref.rmsnorm(x, w, 1e-6)
    q, s = nm.nm_q8_rmsnorm(x.cuda(), w.cuda())
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, norm_limit(1000))


def test_ties_go_to_even(nm):
    """Multiples of 1/2 of a step: a = 127, so the quotients are the values themselves."""
    x = torch.arange(-127, 127.5, 0.5).repeat(2, 1)
    for t in (torch.float32, torch.float16):
        q, s = nm.nm_q8_rows(x.to(t).cuda())
        assert torch.equal(q.cpu(), torch.round(x).to(torch.int8)) and torch.all(s == 1.0)
    # (w = 1: the same through the norm)
    q, _ = nm.nm_q8_rmsnorm(x.cuda(), torch.ones(x.shape[1], device="cuda"))
    assert torch.equal(q.cpu(), torch.round(x).to(torch.int8))


def test_values_next_to_a_border(nm):
    """Numbers a last bit away from the border between two integers, on either side."""
    a = torch.tensor(3.7182817)
    k = torch.arange(0, 126) + 0.5
    mid = (k.double() * a.double() / 127.0).float()
    x = torch.cat([a[None], mid, torch.nextafter(mid, torch.tensor(9.0)), torch.nextafter(mid, torch.tensor(0.0))])[None].repeat(3, 1)
    want, _ = ref.rows(x)
    q, _ = nm.nm_q8_rows(x.cuda())
    assert torch.equal(q.cpu(), want)
    want, _ = ref.rmsnorm(x, torch.full((x.shape[1],), 1.1), 1e-6)
    q, _ = nm.nm_q8_rmsnorm(x.cuda(), torch.full((x.shape[1],), 1.1, device="cuda"))
    assert torch.equal(q.cpu(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("h", [24, 2000, 20000])
def test_rows_that_are_not_finite_zero_or_out_of_range(nm, dtype, h):
    top = torch.finfo(dtype).max
    x = randn(12, h, seed=8, dtype=dtype)
    w = randn(h, seed=9, dtype=dtype)
    x[0] = 0
    x[1, h // 2] = float("nan")
    x[2, h - 1] = float("inf")
    x[3, 0] = -float("inf")
    x[4] = top                                        # squares overflow 32 bits (fp32, bf16)
    x[5] = torch.finfo(dtype).tiny                    # least normal numbers
    x[6] = torch.finfo(dtype).smallest_normal / 4
    x[7] = 0
    x[7, 5] = 1e-7
    x[8] = -top
    want_q, want_s = ref.rmsnorm(x, w, 1e-6)
    q, s = nm.nm_q8_rmsnorm(x.cuda(), w.cuda(), 1e-6)
    bad = ~torch.isfinite(want_s) | (want_s > 3.4e38)
    assert torch.equal(torch.isnan(s.cpu()), bad) and torch.isnan(s.cpu()[1:4]).all()
    assert torch.equal(q.cpu()[~bad], want_q[~bad]) and not q.cpu()[bad].any()
    same_scale(s[~bad.cuda()], want_s[~bad], norm_limit(h))
    want_q, want_s = ref.rows(x)
    q, s = nm.nm_q8_rows(x.cuda())
    bad = ~torch.isfinite(want_s)
    assert torch.equal(torch.isnan(s.cpu()), bad) and torch.equal(q.cpu(), want_q)
    same_scale(s[~bad.cuda()], want_s[~bad], 2.0 ** -24)


def test_silu_mul_far_out(nm):
    """Gates where the exponential leaves 32 bits, products that do, and rows whose products are all tiny."""
    g = torch.tensor([[-95.0, 4.0, -88.5, 90.0, 0.0, -0.0, 1e-35, -3e38], [-100.0, -101.0, -102.5, -99.0, -120.0, -100.5, -98.0, -103.0],
                      [1e30, 2e30, -5.0, 3.0, 0.5, 1.0, 2.0, -1.0], [3e38, 1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 7.0], [-90.0] * 8,
                      [float("-inf")] + [1.0] * 7, [0.0] * 8])
    u = torch.tensor([[1.0, 2.0, 3e38, 1e-3, 5.0, 7.0, 1e30, 1.0], [1.0, 2.0, 3.0, -4.0, 5.0, 1.5, 0.5, 8.0],
                      [1e-30, 1e5, 1.0, 2.0, 3.0, 4.0, 5.0, 6.0], [3e38, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0], [3e38, -1e38, 2e38, 1.0, 0.0, 1e37, 3e37, -3e38],
                      [1.0] * 8, [1.0] * 8])
    want_q, want_s = ref.silu_mul(g, u)
    q, s = nm.nm_q8_silu_mul(g.cuda(), u.cuda())
    bad = ~(want_s <= 3.4e38)
    assert torch.equal(torch.isnan(s.cpu()), bad)
    assert torch.equal(q.cpu()[~bad], want_q[~bad]) and not q.cpu()[bad].any()
    same_scale(s[~bad.cuda()], want_s[~bad], 2.0 ** -24)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_what_lies_around(nm, dtype):
    """Halves of one tensor, rows that are not 16-byte aligned, outputs inside larger buffers that stay as they were."""
    tokens, h = 21, 200
    both = randn(tokens, 2 * h, seed=10, dtype=dtype).cuda()
    gate, up = both[:, :h], both[:, h:]
    want_q, want_s = ref.silu_mul(gate.cpu(), up.cpu())
    q, s = nm.nm_q8_silu_mul(gate, up)
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, 2.0 ** -24)
    odd = randn(tokens, h + 3, seed=11, dtype=dtype).cuda()[:, 1:h + 1]          # every row at another offset
    buf = torch.full((tokens + 2, 256), 77, dtype=torch.int8, device="cuda")
    scales = torch.full((tokens + 2,), -5.0, device="cuda")
    want_q, want_s = ref.rows(odd.cpu())
    q, s = nm.nm_q8_rows(odd, q=buf[1:-1, 16:16 + h], scale=scales[1:-1])
    assert q.data_ptr() == buf[1, 16:].data_ptr() and torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, 2.0 ** -24)
    buf[1:-1, 16:16 + h] = 77
    assert torch.all(buf == 77) and scales[0] == -5.0 and scales[-1] == -5.0


@pytest.mark.parametrize("h", [136, 1001, 20000])
@pytest.mark.parametrize("into", ["residual", "x", "beside"])
def test_residual_in_place(nm, h, into):
    x, r, w = (randn(30, h, seed=12 + i, dtype=torch.bfloat16) for i in range(3))
    w = w[0]
    want_q, want_s, want_r = ref.rmsnorm(x, w, 1e-6, r)
    if into == "beside":
        buf = torch.empty(30, 3 * h, dtype=torch.bfloat16, device="cuda")
        buf[:, :h], buf[:, h:2 * h] = x, r
        xd, rd, out = buf[:, :h], buf[:, h:2 * h], buf[:, 2 * h:]
    else:
        xd, rd = x.cuda(), r.cuda()
        out = rd if into == "residual" else xd
    q, s, got = nm.nm_q8_rmsnorm(xd, w.cuda(), 1e-6, residual=rd, residual_out=out)
    assert got.data_ptr() == out.data_ptr() and torch.equal(out.cpu(), want_r) and torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, norm_limit(h))


def test_one_row_of_anything(nm):
    """A single token's pitch is of no account."""
    x = randn(8, 96, seed=15)[::3].cuda()[:1]
    q, s = nm.nm_q8_rows(x.expand(1, 96))
    want_q, _ = ref.rows(x.cpu())
    assert torch.equal(q.cpu(), want_q)


def test_no_tokens(nm):
    q, s = nm.nm_q8_rows(torch.empty(0, 64, device="cuda"))
    assert q.shape == (0, 64) and s.shape == (0,)
    q, s, r = nm.nm_q8_rmsnorm(torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda"), residual=torch.empty(0, 64, device="cuda"))
    assert r.shape == (0, 64)


def test_refusals(nm):
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    with pytest.raises(nm.NmError) as e:
        nm.nm_q8_rmsnorm(x, w, 0.0)
    assert e.value.status == nm.NM_ERR_INVALID_ARG
    for bad in (lambda: nm.nm_q8_rmsnorm(x, w[:63]), lambda: nm.nm_q8_rmsnorm(x, w, residual=x.half()), lambda: nm.nm_q8_rmsnorm(x, w, residual_out=x),
                lambda: nm.nm_q8_rmsnorm(x, w.double()), lambda: nm.nm_q8_silu_mul(x, x[:3]), lambda: nm.nm_q8_silu_mul(x, x.bfloat16()),
                lambda: nm.nm_q8_rows(x.t()), lambda: nm.nm_q8_rows(x, q=x), lambda: nm.nm_q8_rows(x, scale=x[0])):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(nm.NmError):   # rows on top of each other
        nm.nm_q8_rows(x[:1].expand(4, 64))
    with pytest.raises(nm.NmError):   # rows of q that are no multiple of 16 bytes apart
        nm.nm_q8_rows(x, q=torch.empty(4, 65, dtype=torch.int8, device="cuda")[:, :64])
    with pytest.raises(nm.NmError):   # in place, shifted
        big = torch.zeros(5, 64, device="cuda")
        nm.nm_q8_rmsnorm(big[:4], w, residual=x, residual_out=big[1:])


def test_another_stream_and_a_captured_call(nm):
    x, w = randn(50, 512, seed=16, dtype=torch.bfloat16).cuda(), randn(512, seed=17, dtype=torch.bfloat16).cuda()
    want = nm.nm_q8_rmsnorm(x, w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = nm.nm_q8_rmsnorm(x, w)
    st.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    buf = torch.zeros_like(x)
    q, s = torch.empty_like(want[0]), torch.empty_like(want[1])
    q = torch.empty_strided(want[0].shape, want[0].stride(), dtype=torch.int8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nm.nm_q8_rmsnorm(buf, w, q=q, scale=s)
    buf.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q, want[0]) and torch.equal(s, want[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("h", [1, 5, 13, 100, 511, 1001, 1500, 2047, 3001, 4093, 6001, 8187, 12285, 16379, 16391, 20011, 30001, 40003])
@pytest.mark.parametrize("tokens", [2, 310])
def test_ragged_rows_16_bytes_apart(nm, dtype, h, tokens):
    """Rows that end inside a 16-byte piece but begin on one: all operators, every shape of the kernel."""
    if tokens > 2 and h > 17000:
        tokens = 299
    ld = -(-h // 8) * 8 + 8
    full = [2 * randn(tokens, ld, seed=20 + i, dtype=dtype) for i in range(2)]
    x, r = (t.cuda()[:, :h] for t in full)
    w = randn(h, seed=22, dtype=dtype)
    q, s, out = nm.nm_q8_rmsnorm(x, w.cuda(), 1e-6, residual=r)
    want_q, want_s, want_r = ref.rmsnorm(full[0][:, :h], w, 1e-6, full[1][:, :h])
    assert torch.equal(out.cpu(), want_r) and torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, norm_limit(h))
    q, s = nm.nm_q8_rmsnorm(x, w.cuda(), 1e-6)
    want_q, want_s = ref.rmsnorm(full[0][:, :h], w, 1e-6)
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, norm_limit(h))
    q, s = nm.nm_q8_silu_mul(x, r)
    want_q, want_s = ref.silu_mul(full[0][:, :h], full[1][:, :h])
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, 2.0 ** -24)
    q, s = nm.nm_q8_rows(x)
    want_q, want_s = ref.rows(full[0][:, :h])
    assert torch.equal(q.cpu(), want_q)
    same_scale(s, want_s, 2.0 ** -24)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("h", [40, 600, 4096, 9000])
def test_long_batches_with_rows_out_of_the_ordinary(nm, dtype, h):
    """Blocks that take many rows each, among them padding, rows that are not finite, tiny and huge ones."""
    tokens = 5000 if h < 5000 else 2000
    x, u = randn(tokens, h, seed=30, dtype=dtype), randn(tokens, h, seed=31, dtype=dtype)
    kind = torch.randint(0, 12, (tokens,), generator=torch.Generator().manual_seed(32))
    x[kind == 0] = 0
    x[kind == 1, h // 3] = float("nan")
    x[kind == 2, h - 1] = float("inf")
    x[kind == 3] = torch.finfo(dtype).max
    x[kind == 4] *= 1e-4
    x[kind == 5, 0] = -100.0                         # a gate far out
    u[kind == 6, 1] = 2e4                            # a product that stands out
    w = randn(h, seed=33, dtype=dtype)
    want = [ref.rmsnorm(x, w, 1e-6), ref.silu_mul(x, u), ref.rows(x)]
    got = [nm.nm_q8_rmsnorm(x.cuda(), w.cuda(), 1e-6), nm.nm_q8_silu_mul(x.cuda(), u.cuda()), nm.nm_q8_rows(x.cuda())]
    for (want_q, want_s), (q, s), limit in zip(want, got, (norm_limit(h), 2.0 ** -24, 2.0 ** -24)):
        bad = ~(want_s <= 3.4e38)
        assert torch.equal(torch.isnan(s.cpu()), bad) and not q.cpu()[bad].any()
        assert torch.equal(q.cpu()[~bad], want_q[~bad])
        same_scale(s[~bad.cuda()], want_s[~bad], limit)


def test_calls_on_two_streams_at_once(nm):
    x = [randn(3000, 1000, seed=40 + i, dtype=torch.bfloat16).cuda() for i in range(2)]
    want = [nm.nm_q8_silu_mul(x[i], x[1 - i]) for i in range(2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(8):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(nm.nm_q8_silu_mul(x[i], x[1 - i]))
    torch.cuda.synchronize()
    assert all(torch.equal(q, want[i][0]) and torch.equal(s, want[i][1]) for i in range(2) for q, s in got[i])
