"""The binding where there is more than one device (CPU only: devices are stand-ins)."""
import pytest

from paper_2609_34370_b200 import binding


class _Device:
    def __init__(self, index):
        self.index = index


class _Tensor:
    is_cuda = True

    def __init__(self, index):
        self.device = _Device(index)

    def get_device(self):
        return self.device.index


@pytest.mark.parametrize("how", ["positional", "keyword first", "keyword last", "another tensor first"])
@pytest.mark.parametrize("index", [0, 3])
def test_a_call_is_made_on_the_device_of_its_first_argument(how, index, monkeypatch):
    entered = []

    class Guard:
        def __init__(self, device):
            entered.append(device.index)

        def __enter__(self):
            return self

        def __exit__(self, *exc):
            return False

    class Torch:
        class cuda:
            device = Guard

    monkeypatch.setattr(binding, "torch", Torch)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    call = binding._on_device_of(lambda logits, token_ids=None, top_n=0: (logits, token_ids, top_n))
    x, other = _Tensor(index), None if how != "another tensor first" else _Tensor(7)
    if how == "positional":
        got = call(x, top_n=3)
    elif how == "keyword first":
        got = call(logits=x, top_n=3)
    elif how == "keyword last":
        got = call(top_n=3, logits=x)
    else:
        got = call(token_ids=other, top_n=3, logits=x)
    assert got == (x, other, 3)
    assert entered == ([] if index == 0 else [index])


def test_calls_without_a_device_tensor_reach_their_own_checks():
    call = binding._on_device_of(lambda logits, top_n=0: (logits, top_n))
    assert call(None, 2) == (None, 2) and call(top_n=2, logits="x") == ("x", 2)
    with pytest.raises(TypeError):
        call(top_n=2)
