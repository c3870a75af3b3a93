"""The rotation of 16-bit rows is that of float64 arithmetic, rounded to binary32 and then to 16 bits: to the last bit where an
element nearly cancels, and in the sign of a zero."""
import numpy as np
import pytest
import torch

import paper_2609_34370_b200 as spx

pytestmark = pytest.mark.gpu
DEV = "cuda"

# (position, x0, x1): pair 0 turns by the position itself, and x0 cos - x1 sin cancels to 2^-32 of its terms and further.  Found by a
# search over positions below 2^29 and all pairs of 8-bit mantissas, for results that arithmetic good to 2^-46 of the terms rounds to the
# other side of a border of bfloat16.
NEAR = [(81046462, 70.0, 228.0), (113878523, -252.0, 177.0), (163482650, -308.0, 246.0), (176334560, -171.0, 145.0), (359827317, 298.0, 189.0),
        (398737112, -151.0, 140.0), (451542733, -25.375, 155.0), (466627870, 146.0, 215.0), (469914213, -380.0, 203.0), (518217605, -111.5, 249.0)]


def _bits(x):
    """float64 -> binary32 -> bfloat16, as bits."""
    b = np.asarray(x, np.float64).astype(np.float32).view(np.uint32).astype(np.int64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16).view(np.int16)


def _append(rows, lens, m, q=None, positions=None, d=128):
    pages = -(-max(lens) // 16) + 1
    pool = torch.zeros(len(lens) * pages, 1, 16, d, dtype=torch.bfloat16, device=DEV)
    table = torch.arange(len(lens) * pages, dtype=torch.int32, device=DEV).view(len(lens), pages)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    starts = [0] + np.cumsum(m).tolist()
    extra = {} if positions is None else dict(positions=positions.to(DEV), rope_sections=[d // 2])
    status = spx.kv_append(rows.to(DEV), rows.to(DEV), pool, pool.clone(), pool.stride()[:3], table, ints(lens), ints(starts), 16, len(lens) * pages,
                           rope_base=10000.0, q_rows=q, **extra)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    t = torch.cat([torch.arange(n - k, n) for n, k in zip(lens, m)])
    r = torch.cat([torch.full((k,), i) for i, k in enumerate(m)])
    return pool.cpu()[table.cpu().long()[r, t // 16], 0, t % 16]


@pytest.mark.parametrize("swap", [False, True])
def test_results_that_nearly_cancel(swap):
    """In y0 = x0 cos - x1 sin, and, with x1 and -x0 in the places of x0 and x1, in y1 = x1 cos + x0 sin."""
    n = len(NEAR)
    at = np.array([a for a, _, _ in NEAR], np.longdouble)
    x0, x1 = (np.array([x[i] for x in NEAR], np.float64) for i in (1, 2))
    exact = x0 * np.cos(at) - x1 * np.sin(at)
    # the expected bits do not hang on the last bits of a library's sine and cosine
    room = 2.0 ** -51 * np.maximum(np.abs(x0), np.abs(x1))
    want = _bits(exact.astype(np.float64))
    assert (want == _bits((exact - room).astype(np.float64))).all() and (want == _bits((exact + room).astype(np.float64))).all()
    rows = torch.randn(n, 1, 128, generator=torch.Generator().manual_seed(1)).bfloat16()
    rows[:, 0, 0], rows[:, 0, 64] = torch.from_numpy(-x1 if swap else x0).bfloat16(), torch.from_numpy(x0 if swap else x1).bfloat16()
    q = rows.repeat(1, 3, 1).to(DEV)
    pos = torch.tensor([[a for a, _, _ in NEAR]], dtype=torch.int32)
    kept = _append(rows, [n], [n], q, pos)
    col = 64 if swap else 0
    assert (kept[:, col].view(torch.int16).numpy() == want).all()
    assert (q[:, :, col].cpu().view(torch.int16).numpy() == want[:, None]).all()


def test_zeros_of_either_sign():
    """Elements of zero keep the signs that products and sum in float64 give them, and the row's others their values."""
    lens, m = [40, 23], [40, 5]
    g = torch.Generator().manual_seed(2)
    rows = torch.randn(45, 1, 128, generator=g).bfloat16()
    zero = torch.where(torch.rand(45, 1, 128, generator=g) < 0.5, 0.0, -0.0).bfloat16()
    rows = torch.where(torch.rand(45, 1, 1, generator=g) < 0.7, torch.where(torch.rand(45, 1, 128, generator=g) < 0.6, zero, rows), zero)
    q = rows.clone().to(DEV)
    kept = _append(rows, lens, m, q)
    t = np.concatenate([np.arange(n - k, n) for n, k in zip(lens, m)]).astype(np.float64)
    angle = t[:, None] * 10000.0 ** (-2.0 * np.arange(64) / 128)
    x0, x1 = rows[:, 0, :64].double().numpy(), rows[:, 0, 64:].double().numpy()
    c, s = np.cos(angle), np.sin(angle)
    want = np.concatenate((x0 * c - x1 * s, x1 * c + x0 * s), -1)
    for got in (kept, q[:, 0].cpu()):
        z = want == 0
        assert (np.signbit(got.double().numpy())[z] == np.signbit(want)[z]).all()
        assert (np.abs(got.double().numpy() - want) <= (2.0 ** -8 + 2.0 ** -24) * np.abs(want)).all()


def test_tiny_and_large_rows():
    """Elements near the ends of bfloat16's range: the remainders of their products are below binary32's smallest, or past its largest."""
    g = torch.Generator().manual_seed(3)
    rows = torch.randn(64, 1, 128, generator=g)
    rows[:40] *= 2.0 ** -torch.randint(90, 133, (40, 1, 1), generator=g).double()
    rows[40:] *= 2.0 ** 124
    rows = rows.float().bfloat16()
    kept = _append(rows, [64], [64])
    angle = np.arange(64.0)[:, None] * 10000.0 ** (-2.0 * np.arange(64) / 128)
    x0, x1 = rows[:, 0, :64].double().numpy(), rows[:, 0, 64:].double().numpy()
    want = np.concatenate((x0 * np.cos(angle) - x1 * np.sin(angle), x1 * np.cos(angle) + x0 * np.sin(angle)), -1)
    got = kept.view(torch.int16).numpy()
    # a sine or cosine may differ in its last bit between libraries: values whose bits hang on 2^-51 of their terms are left out
    room = 2.0 ** -51 * np.concatenate((np.hypot(x0, x1),) * 2, -1)
    sure = (_bits(want - room) == _bits(want + room))
    assert sure.mean() > 0.999 and (got == _bits(want))[sure].all()


@pytest.mark.parametrize("base", [10000.0, 1e6])
def test_millions_of_results(base):
    """60,000 rows, eight million results a call: some hundreds lie within two binary32 steps of a border between two bfloat16 values."""
    n = 60000
    g = torch.Generator().manual_seed(4)
    rows = torch.randn(n, 1, 128, generator=g).bfloat16()
    pages = -(-n // 16)
    pool = torch.zeros(pages, 1, 16, 128, dtype=torch.bfloat16, device=DEV)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    x = rows.to(DEV)
    status = spx.kv_append(x, x, pool, pool.clone(), pool.stride()[:3], ints([list(range(pages))]), ints([n]), ints([0, n]), 16, pages, rope_base=base)
    assert int(status.item()) == 0
    angle = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * torch.tensor([base ** (-2.0 * i / 128) for i in range(64)], dtype=torch.float64, device=DEV)
    c, s = torch.cos(angle), torch.sin(angle)
    x0, x1 = x[:, 0, :64].double(), x[:, 0, 64:].double()
    got = pool.view(-1, 128)[:n]
    near = 0
    for y, have in ((x0 * c - x1 * s, got[:, :64]), (x1 * c + x0 * s, got[:, 64:])):
        bits = lambda v: v.float().bfloat16().view(torch.int16)  # noqa: E731
        # (frequency, angle, sine: off by 2^-52 of themselves each between libraries; angles below 2^16)
        room = 2.0 ** -36 * torch.maximum(x0.abs(), x1.abs()) * (angle.abs() * 2.0 ** -16).clamp(min=2.0 ** -14)
        sure = bits(y - room) == bits(y + room)
        assert float(sure.double().mean()) > 0.9999
        assert torch.equal(have.view(torch.int16)[sure], bits(y)[sure])
        near += int((((y.float().view(torch.int32) & 0xFFFF) - 0x8000).abs() <= 2).sum())
    assert near > 200
