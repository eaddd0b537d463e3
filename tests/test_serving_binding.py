"""What the binding of the operators around the step hands to the library, without a GPU: tensors on the
CPU that say they are on a device, and a library that writes its arguments down."""
import pytest

from paper_2608_26004_gb300 import asymspec as A
from paper_2608_26004_gb300 import build
from paper_2608_26004_gb300 import serving as S

torch = pytest.importorskip("torch")


class Placed(torch.Tensor):
    """A tensor that claims to be on cuda:`place`."""
    place = 0

    def get_device(self):
        return self.place


def placed(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Placed)


def ints(*shape):
    return placed(*shape, dtype=torch.int32)


class Library:
    """Writes down each call's name and arguments, and launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return A.OK
        return call


@pytest.fixture
def library(monkeypatch):
    build.build_cuda()
    S._begin()
    fake = Library()
    monkeypatch.setattr(S, "_lib", fake)
    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: Placed.place)
    monkeypatch.setattr(S.torch._C, "_cuda_getCurrentRawStream", lambda dev: 0x5000 + dev, raising=False)
    return fake


def constraints(library):
    (name, args), = library.calls
    assert name == "asymspec_constrain_logits"
    return S.Constraints.from_buffer_copy(args[0])


def test_a_history_that_has_no_room_yet(library):
    lens, prompts = ints(2), ints(2)
    S.constrain_logits(placed(2, 1, 64), history=ints(2, 0), history_len=lens, prompt_len=prompts)
    c = constraints(library)
    assert c.history and c.history_width == 0       # a group that is there: its lengths are looked at
    assert c.history_len == lens.data_ptr() and c.prompt_len == prompts.data_ptr()


def test_no_masks_this_round(library):
    rows = ints(2, 3)
    S.constrain_logits(placed(2, 3, 64), mask=ints(0, 2), mask_rows=rows)
    c = constraints(library)
    assert c.mask and c.mask_count == 0 and c.mask_ld == 2 and c.mask_rows == rows.data_ptr()


def test_a_mask_without_rows_is_no_absent_mask(library):
    with pytest.raises(ValueError):
        S.constrain_logits(placed(2, 3, 64), mask=ints(0, 2))
    assert not library.calls


def test_no_requests(library):
    S.constrain_logits(placed(0, 3, 64), history=ints(0, 5), history_len=ints(0), mask=ints(0, 2),
                       mask_rows=ints(0, 3))
    c = constraints(library)
    assert not (c.history or c.history_len or c.mask or c.mask_rows)
