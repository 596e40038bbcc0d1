"""Quotients within a few roundings of the border between two integers, on either side, the border of 0 and 1 above all: the integers
are those of the definition in 64 bits whichever arithmetic a kernel works its quotients out in."""
import pytest
import torch

import q8_reference as ref

pytestmark = pytest.mark.gpu

# (columns, least tokens) of every shape of the row kernels: a warp to a row, blocks, few and many rows, rows off the 16-byte boundaries, rows
# that are read again
SHAPES = [(96, 1), (1001, 1), (1001, 1000), (2048, 1), (2048, 300), (4096, 300), (4099, 1), (8192, 1), (8192, 300), (12288, 300), (16384, 1), (20000, 1), (20001, 1)]
FP32_OFFSETS = [-40, -12, -5, -3, -2, -1, 0, 1, 2, 3, 5, 12, 40]   # last places of a factor


@pytest.fixture(scope="module")
def nm():
    from paper_2507_17301_b200 import nm as mod
    return mod


def generator(seed):
    return torch.Generator().manual_seed(seed)


def some_k(n, g):
    """Integers below the border at k + 1/2: every second one 0, the others up to 125."""
    return torch.where(torch.rand(n, generator=g) < 0.5, 0, torch.randint(0, 126, (n,), generator=g)).double()


def moved(x, places):
    """fp32 numbers, `places` last places away from zero."""
    return (x.view(torch.int32) + places.int()).view(torch.float32)


def silu(g):
    return g / (1.0 + torch.exp(-g))


def gates_and_ups(n, top_gate, top_up, seed):
    """n fp32 pairs; the first has the largest product, the quotients of the others lie next to a border."""
    g = generator(seed)
    gate = (50.0 * torch.rand(n, generator=g) - 40.0).float()
    gate[::3] = (8.0 * torch.rand(len(gate[::3]), generator=g) - 16.0).float()
    gate[0] = top_gate
    a = silu(gate[0].double()) * torch.tensor(top_up).float().double()
    up = ((some_k(n, g) + 0.5) * a / 127.0 / silu(gate.double()))
    up = moved(up.float(), torch.tensor(FP32_OFFSETS)[torch.randint(0, len(FP32_OFFSETS), (n,), generator=g)])
    up[0] = top_up
    up[(gate.double() * up.double()).abs() > 2.0 ** 39] = 0.0        # (beyond that a row is worked out in 64 bits from the start)
    up[torch.rand(n, generator=g) < 0.5] *= -1.0
    up[0] = top_up
    return gate, up


@pytest.mark.parametrize("h,tokens", SHAPES)
def test_silu_mul(nm, h, tokens):
    tops = [(30.0, 1e-6), (4.0, 2.0), (0.7, 3.0), (-1.1, 40.0), (11.0, 0.5)]
    rows = [gates_and_ups(h, *tops[i % len(tops)], seed=1000 * h + i) for i in range(max(5, 20000 // h))]
    rows = (rows * -(-tokens // len(rows)))[:max(tokens, len(rows))]
    gate, up = (torch.stack(t) for t in zip(*rows))
    want_q, _ = ref.silu_mul(gate, up)
    assert (want_q.abs() <= 1).float().mean() > 0.3
    q, _ = nm.nm_q8_silu_mul(gate.cuda(), up.cuda())
    wrong = q.cpu() != want_q
    assert not wrong.any(), (int(wrong.sum()), gate[wrong][:4], up[wrong][:4], q.cpu()[wrong][:4], want_q[wrong][:4])


def test_silu_mul_of_a_gate_far_below_zero(nm):
    gate, up = torch.tensor([[30.0, -27.427486419677734] + [0.0] * 6]), torch.tensor([[1e-6, 3513.23828125] + [0.0] * 6])
    q, _ = nm.nm_q8_silu_mul(gate.cuda(), up.cuda())
    assert q.cpu()[0, :2].tolist() == [127, -1]


@pytest.mark.parametrize("dtype,within", [(torch.bfloat16, 2e-6), (torch.float16, 1e-6)])
@pytest.mark.parametrize("h", [104, 1001, 4096, 16384, 40000])
def test_silu_mul_of_16_bit_numbers(nm, dtype, within, h):
    """Of all pairs of 16-bit numbers those whose quotient happens to lie next to a border."""
    gates = torch.arange(0, 2 ** 16, dtype=torch.int32).to(torch.int16).view(dtype)
    gates = gates[torch.isfinite(gates) & (gates.float().abs() < 17) & (gates.float().abs() > 2.0 ** -6)]
    found, tops = [], []
    for top_gate, top_up in ((1.3984375, 3.015625), (4.0, 2.0), (6.65625, 1.1484375), (2.28125, 0.80078125), (0.8203125, 5.71875), (9.0625, 3.171875)):
        top = torch.tensor([top_gate, top_up]).to(dtype)
        a = silu(top[0].double()) * top[1].double()
        k = torch.arange(0, 126).double()[:, None]
        up = ((k + 0.5) * a / 127.0 / silu(gates.double())).to(dtype)
        off = (127.0 * silu(gates.double()) * up.double() / a).abs() / (k + 0.5) - 1.0
        at = (off.abs() < within) & torch.isfinite(up)
        g, u = gates.expand_as(up)[at], up[at]
        assert len(g) > 40
        found.append((g, u))
        tops.append(top)
    gate, up = torch.zeros(6, h, dtype=dtype), torch.zeros(6, h, dtype=dtype)
    for row, ((g, u), top) in enumerate(zip(found, tops)):
        n = min(h - 1, len(g))
        gate[row, 1:n + 1], up[row, 1:n + 1] = g[:n], u[:n]
        gate[row, 0], up[row, 0] = top[0], top[1]
    want_q, _ = ref.silu_mul(gate, up)
    q, _ = nm.nm_q8_silu_mul(gate.cuda(), up.cuda())
    wrong = q.cpu() != want_q
    assert not wrong.any(), (int(wrong.sum()), gate[wrong][:4], up[wrong][:4], q.cpu()[wrong][:4], want_q[wrong][:4])


def test_a_norm_next_to_one_half(nm):
    x, w = torch.tensor([[79.13716, 0.3830098]]), torch.tensor([1.5684186, 1.2758478])
    assert 0.5 < 127.0 * x[0, 1].double() * w[1].double() / (x[0, 0].double() * w[0].double()) < 0.50000001
    q, _ = nm.nm_q8_rmsnorm(x.cuda(), w.cuda(), 1e-6)
    assert q.cpu().tolist() == [[127, 1]]


def worst_tops(dtype, seed):
    """Largest elements (s, weight) whose 127 / a is furthest off in 32 bits, three too low and three too high."""
    g = generator(seed)
    s, w = (20.0 + 80.0 * torch.rand(20000, generator=g)).to(dtype).float(), 1.0 + torch.rand(20000, generator=g)
    inv = 127.0 * (1.0 / (s * w))
    off = inv.double() * s.double() * w.double() / 127.0 - 1.0
    order = off.argsort()
    pick = torch.cat([order[:3], order[-3:]])
    return list(zip(s[pick].tolist(), w[pick].tolist()))


@pytest.mark.parametrize("h,tokens", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("residual", [False, True])
def test_norms_with_fp32_weights(nm, h, tokens, dtype, residual):
    for i, (top_s, top_w) in enumerate(worst_tops(dtype, 7)):
        g = generator(100 * h + i)
        s = (torch.exp(torch.randn(h, generator=g)) * 2.0).to(dtype)
        s[0] = top_s
        a = s[0].double() * torch.tensor(top_w).float().double()
        w = ((some_k(h, g) + 0.5) * a / 127.0 / s.double()).float()
        w = moved(w, torch.tensor(FP32_OFFSETS)[torch.randint(0, len(FP32_OFFSETS), (h,), generator=g)])
        w[0] = top_w
        # rows of the same quotients: times powers of two
        x = s.float()[None] * 2.0 ** (torch.arange(max(tokens, 3)) % 5 - 2.0)[:, None]
        x = x.to(dtype)
        r = (x.float() / 2).to(dtype) if residual else None              # (halves are exact, and so is their sum)
        want_q = ref.rmsnorm(r if residual else x, w, 1e-6, r)[0]
        got = nm.nm_q8_rmsnorm((r if residual else x).cuda(), w.cuda(), 1e-6, residual=r.cuda() if residual else None)
        wrong = got[0].cpu() != want_q
        assert not wrong.any(), (int(wrong.sum()), got[0].cpu()[wrong][:4], want_q[wrong][:4])


@pytest.mark.parametrize("h", [96, 1001, 4096, 20000])
def test_plain_rows_of_fp32_numbers(nm, h):
    g = generator(h)
    x = torch.zeros(5, h)
    for i in range(5):
        x[i, 0] = 1.0 + 5.0 * torch.rand(1, generator=g)
        mid = (some_k(h - 1, g) + 0.5) * x[i, 0].double() / 127.0
        x[i, 1:] = moved(mid.float(), torch.tensor(FP32_OFFSETS)[torch.randint(0, len(FP32_OFFSETS), (h - 1,), generator=g)])
    want_q, _ = ref.rows(x)
    q, _ = nm.nm_q8_rows(x.cuda())
    assert torch.equal(q.cpu(), want_q)
