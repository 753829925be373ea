"""Edges of the operators around the linears, without a GPU: what the binding
hands to the library (tensors on the CPU stand in for the GPU's, the library's
call for a function that looks at its arguments), and refusals."""
import contextlib
import ctypes

import pytest
import torch

import paper_2604_06916_amd as sol
from paper_2604_06916_amd import _binding as B

OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE = 0, -1, -2, -3, -4


class HostStream:
    cuda_stream = 0


@pytest.fixture()
def host(monkeypatch):
    """CPU tensors pass for GPU tensors."""
    monkeypatch.setattr(B, "_is_gpu", lambda t: True)
    monkeypatch.setattr(B, "_stream", lambda stream, device: HostStream())
    monkeypatch.setattr(torch.cuda, "stream", lambda st: contextlib.nullcontext())


# ---- the table's frequencies ----------------------------------------------

@pytest.mark.parametrize("view", [lambda b: b[:24], lambda b: b[::2], lambda b: b[5:6].expand(24), lambda b: b[3:3].clone()])
def test_table_frequencies_of_any_stride(host, monkeypatch, view):
    """The library reads `pairs` doubles from the address it is given: they
    have to be the tensor's elements whatever its stride is."""
    f = view(torch.arange(48, dtype=torch.float64) + 1)
    seen = []

    def table(positions, rows, frequencies, pairs, *rest):
        seen.extend((ctypes.c_double * pairs).from_address(frequencies.value) if pairs else [])
        return OK
    monkeypatch.setattr(B.lib, "solfp4_rotary_table", table)
    sol.rotary_table(f, torch.arange(3))
    assert seen == f.tolist()


# ---- the table's device ---------------------------------------------------

@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_table_refuses_other_devices(host, monkeypatch, device):
    """With a stream given nothing else looks at the device: the table would
    be host memory, which the kernel cannot write."""
    calls = []
    monkeypatch.setattr(B.lib, "solfp4_rotary_table", lambda *a: calls.append(a) or OK)
    with pytest.raises(ValueError):
        sol.rotary_table(sol.rotary_frequencies(8), 4, device=device, stream=HostStream())
    assert not calls


def test_table_device_without_an_index_is_the_current_one(host, monkeypatch):
    """out lives on "cuda:1": "cuda" names the same device while it is the current one."""
    class Table(torch.Tensor):
        device = torch.device("cuda", 1)

    class Frequencies(torch.Tensor):
        def to(self, dev):
            assert dev == torch.device("cuda", 1)
            return self
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(B.lib, "solfp4_rotary_table", lambda *a: OK)
    out = torch.empty(4, 8).as_subclass(Table)
    f = sol.rotary_frequencies(8).as_subclass(Frequencies)
    assert sol.rotary_table(f, 4, device="cuda", out=out) is out
    assert sol.rotary_table(f, 4, out=out) is out
