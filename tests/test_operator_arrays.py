"""What the holder refuses of the arrays of a decode step with weights before the library is called.  No GPU: a holder without a
handle, on host tensors, whose library only counts its calls."""
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_abi import good

N, B, HQ, H, D, CAP = 2, 3, 4, 2, 64, 500


class Elsewhere(torch.Tensor):
    """Says that it is on a fourth card."""
    def get_device(self): return 3
    device = property(lambda self: torch.device("cuda", 3))


@pytest.fixture
def holder(monkeypatch):
    """(holder, calls): two layers per call, bf16 rows; "its device" is where host tensors are."""
    calls = []

    class Library:
        @staticmethod
        def madakv_decode_attn_weights(*args):
            calls.append(args)
            return 0

    class Device:
        index = -1                                      # (what a host tensor's get_device() says)

        def __eq__(self, other): return other == torch.device("cpu")
        def __ne__(self, other): return not self == other

    eng = MB.MadaKV.__new__(MB.MadaKV)
    eng.cfg = good(n_layers=N, batch=B, n_q_heads=HQ, n_kv_heads=H, head_dim=D)
    eng.h, eng.tdtype, eng._out_dtype, eng._device, eng.capacity = None, torch.bfloat16, torch.float32, Device(), CAP
    eng._out_row, eng._heads, eng._kv_row = B * HQ * D, B * H, B * H * D
    eng.k_c = eng.v_c = eng.weights_ws = torch.zeros(16, dtype=torch.uint8)
    eng.kv_off, eng.kv_len, eng.kept_idx = torch.zeros(N, B, H, dtype=torch.int64), torch.zeros(N, B, H, dtype=torch.int32), torch.zeros(CAP, dtype=torch.int32)
    monkeypatch.setattr(MB, "lib", lambda: Library)
    monkeypatch.setattr(MB.MadaKV, "_own_stream", lambda self: 0)
    return eng, calls


def step(eng, n=N, **kw):
    bf = torch.bfloat16
    x = dict(q=torch.zeros(n, B, HQ, D, dtype=bf), k_new=torch.zeros(n, B, H, D, dtype=bf), v_new=torch.zeros(n, B, H, D, dtype=bf),
             out=torch.zeros(n, B, HQ, D), acc_in=torch.zeros(CAP), acc_out=torch.zeros(CAP))
    x.update(kw)
    eng.decode_attn_weights(0, n, **x)


def test_arrays_that_fit(holder):
    eng, calls = holder
    step(eng)
    step(eng, k_new=None, v_new=None)
    step(eng, n=1)
    step(eng, n=1, q=torch.zeros(N, B, HQ, D, dtype=torch.bfloat16))           # (more than the call takes)
    assert len(calls) == 4


@pytest.mark.parametrize("name,heads", [("q", HQ), ("k_new", H), ("v_new", H)])
@pytest.mark.parametrize("how", ["layers", "heads", "float", "half", "elsewhere"])
def test_arrays_of_the_step_that_do_not_fit(holder, name, heads, how):
    eng, calls = holder
    x = torch.zeros(N, B, heads, D, dtype=torch.bfloat16)
    x = dict(layers=x[:1], heads=x[:, :, :-1].contiguous(), float=x.float(), half=x.half(), elsewhere=x.as_subclass(Elsewhere))[how]
    with pytest.raises(ValueError, match=name):
        step(eng, **{name: x})
    assert not calls


def test_output_elsewhere(holder):
    eng, calls = holder
    with pytest.raises(ValueError, match="out"):
        step(eng, out=torch.zeros(N, B, HQ, D).as_subclass(Elsewhere))
    assert not calls
