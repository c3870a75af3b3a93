"""The pieces that the attention over 8-bit pools cuts its queries and weights into, over every pattern (CPU: the arithmetic of
csrc/attn_e4m3.cuh restated in torch)."""
import torch


def cut_weight(x):
    """A binary16 value as three e5m2 pieces: the upper byte of it, of what is left, and of what is then left, rounded to nearest."""
    def upper(h):
        return (h.view(torch.int16) & -256).view(torch.float16)
    p1 = upper(x)
    p2 = upper(x - p1)
    p3 = (x - p1 - p2).to(torch.float8_e5m2).to(torch.float16)
    return p1.double() + p2.double() + p3.double()


def weight_error():
    """(largest, root mean square) of the relative error of a weight above the format's least steps, its rounding to binary16 included."""
    fine = 1 + torch.arange(1 << 16, dtype=torch.float64) / (1 << 16) + 2.0 ** -17
    e = (cut_weight((fine * 16).half()) / 16 - fine).abs() / fine
    return e.max().item(), e.square().mean().sqrt().item()


def test_a_weight_is_off_by_two_to_the_minus_nine():
    x = torch.arange(0, 0x7C00, dtype=torch.int32).to(torch.int16).view(torch.float16)
    e = (cut_weight(x) - x.double()).abs()
    # three significant bits cut off, three more, three rounded to nearest: half a step of the ninth, 2^-9, less a little since what is
    # rounded off lies above a leading one
    normal = x >= 2.0 ** -7
    assert (e[normal] <= 2.0 ** -9 * x[normal].double()).all() and (e[normal] > 2.0 ** -9.3 * x[normal].double()).any()
    # below it half the least step of e5m2
    assert (e <= torch.maximum(2.0 ** -9 * x.double(), torch.tensor(2.0 ** -17, dtype=torch.float64))).all()
    largest, rms = weight_error()
    assert largest < 2.0 ** -9 + 2.0 ** -11 and 2.0 ** -11 < rms < 2.0 ** -10.9
    assert (cut_weight(torch.tensor([0.0, 1.0, 65504.0], dtype=torch.float16)) - torch.tensor([0.0, 1.0, 65504.0]).double()).abs().max() <= 128


def test_a_query_element_is_exact_down_to_two_to_the_minus_thirteen_of_the_largest():
    mantissa = torch.arange(128, 256, dtype=torch.float64)
    for below in range(0, 40):                       # the row's largest element lies in [2^7, 2^8)
        x = mantissa * 2.0 ** -below
        h = x.half()
        first = h.to(torch.float8_e4m3fn).half()
        second = (h - first).to(torch.float8_e5m2).half()
        e = (first.double() + second.double() - x).abs().max().item()
        assert e == 0 if below <= 13 else e <= 2.0 ** 7 * 2.0 ** -21, (below, e)
