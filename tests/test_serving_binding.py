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


def every_call(dev_of):
    """Each operator once, on tensors that claim to be on cuda:`dev_of`."""
    cache = placed(3, 16, 2, 64)
    k, slots = placed(4, 2, 64), placed(4, dtype=torch.int64)
    attend = S.CacheAttend.__new__(S.CacheAttend)
    attend.B_max, attend.Q_max, attend.heads, attend.kv_heads, attend.head_dim = 2, 3, 4, 2, 64
    attend.nbytes, attend.workspace, attend.device_index, attend.scale = 256, placed(64), dev_of, 1.0
    return {
        "asymspec_constrain_logits": lambda: S.constrain_logits(placed(2, 3, 64)),
        "asymspec_cache_plan": lambda: S.cache_plan(ints(2), ints(2, 3), ints(2), ints(5), ints(1), block_size=16,
                                                    grow=3),
        "asymspec_cache_write": lambda: S.cache_write(k, k, cache, cache, slots),
        "asymspec_cache_attend": lambda: attend(placed(2, 3, 4, 64), cache, cache, ints(2, 3), ints(2)),
    }


@pytest.mark.parametrize("where", [0, 1])
@pytest.mark.parametrize("name", [n for n in A.EXPORTED if n in (
    "asymspec_constrain_logits", "asymspec_cache_plan", "asymspec_cache_write", "asymspec_cache_attend")])
def test_tensors_on_another_device_than_the_current_one(library, monkeypatch, name, where):
    """A launch goes to the current device: on tensors of another one it is refused, and goes to
    their device's stream where that is the current one."""
    monkeypatch.setattr(Placed, "place", where)
    call = every_call(where)[name]
    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: 1 - where)
    with pytest.raises(ValueError, match="cuda:%d" % where):
        call()
    assert not library.calls
    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: where)
    call()
    (got, args), = library.calls
    assert got == name and args[-1] == 0x5000 + where


def test_a_workspace_on_device_0_that_is_not_the_current_one(library, monkeypatch):
    asked = []
    library.asymspec_cache_attend_workspace_bytes = lambda *a: 256

    def empty(n, dtype, device):
        asked.append(torch.device(device))
        return placed(n, dtype=dtype)

    monkeypatch.setattr(S.torch, "empty", empty)
    for device in (0, "cuda:0", torch.device("cuda", 0), 1, None):
        S.CacheAttend(2, 3, 4, 2, 64, device=device)
    # ("cuda" alone is the current device)
    assert [d.index for d in asked] == [0, 0, 0, 1, None]


class StepTensor(Placed):
    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", Placed.place)


@pytest.mark.parametrize("where", [0, 1])
@pytest.mark.parametrize("name", ["asymspec_fuse_verify_ex", "asymspec_draft_sample"])
def test_the_step_and_the_draw_on_another_device_than_the_current_one(library, monkeypatch, name, where):
    monkeypatch.setattr(A, "_lib", library)
    monkeypatch.setattr(Placed, "place", where)
    z = torch.zeros(2, 3, 64).as_subclass(StepTensor)
    out = {n: torch.zeros(2, dtype=torch.int32) for n in ("accept_len", "next_token", "error_word")}
    step = A.FuseVerify(2, 2)
    step.workspace, step.V_ws, step.nbytes = torch.zeros(64), 64, 256

    def call():
        if name == "asymspec_draft_sample":
            A.draft_tokens(z, out=(out["accept_len"], out["next_token"]))
        else:
            step(z, z, z, ints(2, 2), out=out)

    def launched():
        return [c for c in library.calls if c[0] == name]

    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: 1 - where)
    with pytest.raises(ValueError, match="cuda:%d" % where):
        call()
    assert not launched()
    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: where)
    call()
    (_, args), = launched()
    assert args[-1] == 0x5000 + where


def test_the_steps_workspace_on_device_0_that_is_not_the_current_one(library, monkeypatch):
    asked = []
    monkeypatch.setattr(A, "_lib", library)
    monkeypatch.setattr(A, "workspace_bytes", lambda *a: 256)
    monkeypatch.setattr(S.torch, "zeros", lambda n, dtype, device: asked.append(torch.device(device)))
    for device in (0, "cuda:0", 1, None):
        A.FuseVerify(2, 2, device=device, V_max=64)
    assert [d.index for d in asked] == [0, 0, 1, None]


TOP = 2 ** 31 - 1


@pytest.mark.parametrize("given,passed", [(0, 0), (7, 7), (TOP, TOP), (2 ** 31, TOP), (2 ** 32 + 5, TOP),
                                          (2 ** 63 - 1, TOP), (-1, -1), (-2 ** 32, -1), (-2 ** 31 - 5, -1)])
def test_numbers_past_32_bits_are_not_cut(library, given, passed):
    """C integers take the low bits of a larger number: a window of 2^32 + 5 is not one of 5."""
    cache = placed(3, 16, 2, 64)
    attend = S.CacheAttend.__new__(S.CacheAttend)
    attend.B_max, attend.Q_max, attend.heads, attend.kv_heads, attend.head_dim = 2, 3, 4, 2, 64
    attend.nbytes, attend.workspace, attend.device_index, attend.scale = 256, placed(64), 0, 1.0
    attend(placed(2, 3, 4, 64), cache, cache, ints(2, 3), ints(2), window=given)
    assert library.calls[0][1][11] == passed
    S.cache_plan(ints(2), ints(2, 3), ints(2), ints(5), ints(1), block_size=given, grow=given, capacity=4)
    args = library.calls[1][1]
    assert args[3] == passed and args[5] == passed
