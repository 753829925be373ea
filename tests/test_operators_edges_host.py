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


# ---- overlaps -------------------------------------------------------------

def at(n):
    return ctypes.c_void_p(0x7F0000000000 + n)


def apart(i):
    return at(i << 32)


#: what a call that passes every check gives without a GPU: the launch's error
PASSED = -5

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that passes would launch on addresses that no GPU holds")


def rotate(q=apart(0), qo=apart(1), k=apart(2), ko=apart(3), table=apart(8), pos=None, token=4096, head=512, out_token=4096,
           out_head=512, heads=8, k_heads=8, tokens=6, dim=128, rows=16):
    """In bytes of FP32 elements."""
    return sol.lib.solfp4_rotary(2, 0, 0, q, token // 4, head // 4, qo, out_token // 4, out_head // 4, heads, k, token // 4,
                                 head // 4, ko, out_token // 4, out_head // 4, k_heads, table, rows, pos, 8 if pos else 0,
                                 tokens, dim, dim, None)


@no_gpu
def test_rotary_side_by_side_is_apart():
    """q and k of one packed buffer, in place and as outputs: by tokens
    [tokens, 3, heads, dim], by heads [tokens, heads, 3, dim], heads first
    [heads, tokens, 3, dim] and [3, heads, tokens, dim]."""
    for token, head, k_at in ((3 * 4096, 512, 4096), (3 * 4096, 1536, 512), (1536, 6 * 1536, 512), (512, 6 * 512, 8 * 6 * 512)):
        layout = dict(token=token, head=head, out_token=token, out_head=head)
        assert rotate(q=at(0), qo=at(0), k=at(k_at), ko=at(k_at), **layout) == PASSED
        assert rotate(qo=at(0), ko=at(k_at), q=apart(4), k=apart(5), **layout) == PASSED
        # one element less far apart
        assert rotate(q=at(0), qo=at(0), k=at(k_at - 4), ko=at(k_at - 4), **layout) == EINVAL
        assert rotate(qo=at(0), ko=at(k_at - 4), q=apart(4), k=apart(5), **layout) == EINVAL


@no_gpu
def test_rotary_outputs_over_each_other_are_refused():
    assert rotate() == PASSED
    assert rotate(qo=apart(3)) == EINVAL and rotate(ko=at((1 << 32) + 512)) == EINVAL
    assert rotate(ko=at((1 << 32) + 6 * 4096 - 512)) == EINVAL and rotate(ko=at((1 << 32) + 6 * 4096)) == PASSED
    # in place, k over q
    assert rotate(qo=apart(0), ko=apart(0)) == EINVAL and rotate(qo=apart(0), ko=apart(2)) == PASSED
    assert rotate(qo=apart(2), ko=apart(0)) == EINVAL


@no_gpu
def test_rotary_outputs_over_table_or_positions_are_refused():
    assert rotate(table=apart(1)) == EINVAL and rotate(table=at((3 << 32) + 6 * 4096 - 4)) == EINVAL
    assert rotate(pos=apart(3)) == EINVAL and rotate(pos=apart(9)) == PASSED
    assert rotate(table=at((1 << 32) + 6 * 4096)) == PASSED


W = 64   # columns, FP32


def norm(x=apart(0), xs=W, r=apart(1), rs=W, g=apart(2), gs=W, groups=2, s=apart(3), ss=W, out=apart(4), os=W, rows=6):
    return sol.lib.solfp4_add_rmsnorm(2, x, xs, r, rs, g, gs, groups, 1e-6, s, ss, out, os, rows, W, None)


def back(dy=apart(0), dys=W, x=apart(1), xs=W, g=apart(2), gs=W, ds=apart(3), dss=W, dx=apart(4), dxs=W, dg=apart(5),
         ws=apart(6), wsb=1 << 20, rows=6, groups=2):
    return sol.lib.solfp4_rmsnorm_backward(2, dy, dys, x, xs, g, gs, groups, ds, dss, 1e-6, dx, dxs, dg, ws, wsb, rows, W,
                                           None)


@no_gpu
def test_norm_columns_of_one_buffer_are_apart():
    """Operands that are columns of one [rows, 5 W] buffer, gains columns of a [groups, 2 W] one."""
    at_ = [at(4 * W * i) for i in range(5)]
    s = dict(xs=5 * W, rs=5 * W, ss=5 * W, os=5 * W)
    assert norm() == PASSED
    assert norm(x=at_[0], r=at_[1], s=at_[2], out=at_[3], **s) == PASSED
    assert norm(x=at_[0], r=at_[1], s=at_[1], out=at_[0], **s) == PASSED
    assert norm(x=at_[0], r=at_[1], s=at_[2], out=at_[3], g=at_[4], gs=5 * W, **s) == PASSED
    s = dict(dys=5 * W, xs=5 * W, dss=5 * W, dxs=5 * W)
    assert back(dy=at_[0], x=at_[1], ds=at_[2], dx=at_[3], **s) == PASSED
    assert back(dy=at_[0], x=at_[1], ds=at_[2], dx=at_[2], **s) == PASSED


@no_gpu
def test_norm_columns_over_each_other_are_refused():
    at_ = [at(4 * W * i) for i in range(5)]
    s = dict(xs=5 * W, rs=5 * W, ss=5 * W, os=5 * W)
    one = at(4 * W * 3 - 4)
    assert norm(x=at_[0], r=at_[1], s=at_[2], out=one, **s) == EINVAL
    assert norm(x=at_[0], r=at_[2], s=at_[4], out=one, **s) == EINVAL
    assert norm(x=at_[0], r=at_[4], s=one, out=at_[1], g=at_[2], gs=5 * W, **s) == EINVAL
    assert norm(x=at_[2], r=at_[4], s=one, out=at_[0], **s) == EINVAL
    # rows of another stride meet sooner or later; a last column reaches into the next row's first
    assert norm(x=at_[0], out=at_[2], xs=5 * W, os=4 * W) == EINVAL
    assert norm(x=at_[0], out=at(4 * (4 * W + 1)), xs=5 * W, os=5 * W) == EINVAL
    # one row: its stride does not matter
    assert norm(x=at_[0], out=at_[0], xs=5 * W, os=W, rows=1, groups=1) == PASSED
    s = dict(dys=5 * W, xs=5 * W, dss=5 * W, dxs=5 * W)
    for d in (dict(dy=at_[2]), dict(x=at_[2]), dict(ds=at_[2])):
        assert back(**{**dict(dy=apart(0), x=apart(1), ds=apart(3)), **d}, dx=one, **s) == EINVAL
    assert back(g=at_[2], gs=5 * W, dx=one, dxs=5 * W) == EINVAL


@no_gpu
@pytest.mark.parametrize("pack", [1, 2])
def test_norm_codes_and_scales_over_operands_are_refused(pack):
    fn = sol.lib.mxfp8_add_rmsnorm if pack == 1 else sol.lib.mxfp4_add_rmsnorm
    rows, codes_bytes, scales_bytes = 48, 48 * W // pack, 48 * W // 32

    def call(codes=apart(5), scales=apart(6), x=apart(0), xs=W, r=apart(1), g=apart(2), s=apart(3)):
        return fn(2, x, xs, r, W, g, W, 2, 1e-6, s, W, codes, scales, rows, W, None)
    assert call() == PASSED
    last = 4 * W * rows - 16      # the operands' last 16 bytes
    for i, n in ((0, last), (1, last), (2, 4 * W * 2 - 16), (3, last)):
        assert call(codes=apart(i)) == EINVAL and call(scales=apart(i)) == EINVAL
        assert call(codes=at((i << 32) + n)) == EINVAL and call(codes=at((i << 32) + n + 16)) == PASSED
        assert call(scales=at((i << 32) + n)) == EINVAL and call(scales=at((i << 32) + n + 16)) == PASSED
    assert call(scales=apart(5)) == EINVAL and call(scales=at((5 << 32) + codes_bytes - 16)) == EINVAL
    assert call(scales=at((5 << 32) + codes_bytes)) == PASSED
    assert call(codes=at((6 << 32) + scales_bytes - 16)) == EINVAL and call(codes=at((6 << 32) + scales_bytes + 16)) == PASSED
    # without a residual nothing is written to the sum's address, which then does not matter
    assert fn(2, apart(0), W, None, 0, None, 0, 1, 1e-6, apart(5), W, apart(5), apart(6), rows, W, None) == PASSED


@no_gpu
def test_gradient_outputs_and_workspace_over_operands_are_refused():
    rows = 6
    need = sol.rmsnorm_backward_workspace_bytes(rows, W, 2)
    last = 4 * W * rows - 16
    assert back() == PASSED and back(dg=None) == PASSED
    for i, n in ((0, last), (1, last), (2, 4 * W * 2 - 16), (3, last), (4, last)):
        assert back(dg=apart(i)) == EINVAL and back(ws=apart(i)) == EINVAL
        assert back(dg=at((i << 32) + n)) == EINVAL and back(dg=at((i << 32) + n + 16)) == PASSED
        assert back(ws=at((i << 32) + n)) == EINVAL and back(ws=at((i << 32) + n + 16)) == PASSED
        # the workspace is ignored where there is no gradient of the gain
        assert back(dg=None, ws=apart(i)) == PASSED
    assert back(ws=apart(5)) == EINVAL and back(ws=at((5 << 32) + 2 * W * 4 - 16)) == EINVAL
    assert back(ws=at((5 << 32) + 2 * W * 4)) == PASSED
    assert back(dg=at((6 << 32) + need - 4)) == EINVAL and back(dg=at((6 << 32) + need)) == PASSED
    # in place is still in place
    assert back(dx=apart(0)) == PASSED and back(dx=apart(1)) == PASSED and back(dx=apart(3)) == PASSED
    assert back(dx=apart(2)) == EINVAL


@no_gpu
@pytest.mark.parametrize("kind", ["nvfp4", "mxfp4", "mxfp8"])
def test_linear_output_over_operands_is_refused(kind):
    M, N, K = 8, 32, 64

    def call(out=apart(6), bias=apart(5)):
        if kind == "nvfp4":
            return sol.lib.nvfp4_weight_linear(apart(0), apart(2), apart(3), apart(4), bias, out, M, N, K, None)
        if kind == "mxfp4":
            return sol.lib.mxfp4_weight_linear(apart(0), apart(2), apart(3), bias, out, M, N, K, None)
        return sol.lib.mxfp8_linear(apart(0), apart(1), apart(2), apart(3), bias, out, M, N, K, None)
    assert call() == PASSED
    sizes = {0: M * K * (1 if kind == "mxfp8" else 2), 2: N * K // 2, 3: N * K // (16 if kind == "nvfp4" else 32), 5: N * 2}
    if kind == "mxfp8":
        sizes[1] = M * K // 32
    for i, n in sizes.items():
        assert call(apart(i)) == EINVAL and call(at((i << 32) + n - 16)) == EINVAL and call(at((i << 32) + n)) == PASSED
        assert call(at((i << 32) - M * N * 2)) == PASSED
    if kind == "nvfp4":
        assert call(apart(4)) == EINVAL and call(at((4 << 32) + 16)) == PASSED
    assert call(apart(5), None) == PASSED


@no_gpu
def test_table_over_positions_or_frequencies_is_refused():
    def call(out=apart(2), pos=apart(3)):
        return sol.lib.solfp4_rotary_table(pos, 8, apart(1), 16, None, 1, 1.0, out, None)
    assert call() == PASSED and call(pos=None) == PASSED
    for i, n in ((1, 16 * 8), (3, 8 * 8)):
        assert call(apart(i)) == EINVAL and call(at((i << 32) + n - 4)) == EINVAL and call(at((i << 32) + n)) == PASSED
    assert call(apart(3), None) == PASSED


def test_rotary_sizes_beyond_the_stated_ones_are_refused():
    def call(heads=1, dim=64, tokens=4):
        return sol.lib.solfp4_rotary(0, 0, 0, apart(0), heads * dim, dim, apart(1 << 8), heads * dim, dim, heads, None, 0, 0,
                                     None, 0, 0, 0, apart(1 << 10), 16, None, 0, tokens, dim, 64, None)
    assert call(heads=1 << 20) == ESHAPE and call(dim=1 << 20) == ESHAPE and call(tokens=1 << 31) == ESHAPE
    assert call(heads=1 << 16, dim=1 << 15) == ESHAPE
