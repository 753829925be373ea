"""The operators around the linears at sizes past 2^31 elements, 4 GiB and the
2^32 threads that one launch may have.  The whole outputs are far beyond a
CPU oracle: sampled rows (first, last, around every 4 GiB of a buffer and
around every 2^32 threads) are compared bit for bit with the same rows in a
small call, which other tests hold against float64."""
import numpy as np
import pytest
import torch

import paper_2604_06916_amd as sol
from gpu_util import device, say

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def sample(rows, row_bytes, per_launch=None):
    """Rows to look at, as a device tensor; per_launch: rows of 2^32 threads."""
    at = {0, 1, rows - 2, rows - 1}
    for step in ((1 << 32) / row_bytes, per_launch):
        n = 1
        while step and n * step < rows:
            at |= {int(n * step) + d for d in range(-5, 6)}
            n += 1
    return torch.tensor(sorted(r for r in at if 0 <= r < rows), device=device())


def test_norm_past_a_launch():
    """Four rows a workgroup of 256 threads: 2^26 rows are 2^32 threads."""
    rows, width = (1 << 26) + 5, 264
    x = torch.empty((rows, width), dtype=torch.bfloat16, device=device())
    x.normal_(generator=torch.Generator(device=device()).manual_seed(1))
    say(f"  norm of {rows} x {width} ({rows * width * 2 / 2**30:.1f} GiB) in place")
    at = sample(rows, 2 * width, 1 << 26)
    want, _ = sol.add_rmsnorm(x[at])
    out, _ = sol.add_rmsnorm(x, out=x)
    assert out is x and torch.equal(x[at], want)
    # every row's mean square is 1, but for its BF16 rounding
    for i in range(0, rows, 1 << 24):
        q = x[i:i + (1 << 24)].float().square_().mean(1)
        assert float((q - 1).abs().max()) < 2.0 ** -6


@pytest.mark.parametrize("kind", ["mxfp8", "mxfp4"])
def test_quantized_norm_past_a_launch(kind):
    rows, width = (1 << 26) + 5, 288
    one = torch.randn(1, width, generator=torch.Generator().manual_seed(2)).bfloat16().to(device())
    call = getattr(sol, f"{kind}_add_rmsnorm")
    want = call(one)
    codes = torch.zeros((rows, want[0].shape[1]), dtype=torch.uint8, device=device())
    scales = torch.zeros((rows, width // 32), dtype=torch.uint8, device=device())
    say(f"  {kind} norm of {rows} equal rows ({codes.numel() / 2**30:.1f} GiB of codes)")
    call(one.expand(rows, width), codes=codes, scales=scales)
    for i in range(0, rows, 1 << 24):
        assert bool((codes[i:i + (1 << 24)] == want[0]).all()) and bool((scales[i:i + (1 << 24)] == want[1]).all())


def test_gradients_past_4gib():
    rows, width, groups = (1 << 20) + 6, 2080, 2
    g = torch.Generator(device=device()).manual_seed(3)
    dy, x = (torch.empty((rows, width), dtype=torch.bfloat16, device=device()).normal_(generator=g) for _ in range(2))
    gain = torch.randn(groups, width, device=device(), generator=g).bfloat16()
    say(f"  gradients of {rows} x {width} ({rows * width * 2 / 2**30:.1f} GiB)")
    at = sample(rows, 2 * width)
    at = torch.cat((at, torch.tensor([rows // 2 - 1, rows // 2], device=device())))
    # each sampled row with its own gain
    per_row = gain[at // (rows // groups)]
    want, _ = sol.rmsnorm_backward(dy[at], x[at], per_row)
    sums = torch.zeros(groups, width, dtype=torch.float64, device=device())
    terms = torch.zeros_like(sums)
    step = rows // groups // 11 + 1
    for i in range(groups):
        for a in range(i * (rows // groups), (i + 1) * (rows // groups), step):
            b = min(a + step, (i + 1) * (rows // groups))
            s = x[a:b].float()
            n = dy[a:b].float() * s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-6)
            sums[i] += n.sum(0, dtype=torch.float64)
            terms[i] += n.abs().sum(0, dtype=torch.float64)
    dx, dgain = sol.rmsnorm_backward(dy, x, gain, dx=dy)
    assert dx is dy and torch.equal(dy[at], want)
    # FP32 sums of the kernel's 2^-18 terms in partial sums of at most 2^12 rows, then 2^9 parts
    assert bool(((dgain.double() - sums).abs() <= terms * (2.0 ** -17 + (2 ** 12 + 2 ** 9) * 2.0 ** -24)).all())


def test_rotary_past_a_launch():
    """A head of 33 pieces of 16 bytes takes a wave: 2^26 tokens of one head are 2^32 threads."""
    tokens, dim = (1 << 26) + 5, 251
    q = torch.empty((tokens, 1, dim), dtype=torch.bfloat16, device=device())
    q.normal_(generator=torch.Generator(device=device()).manual_seed(4))
    table = sol.rotary_table(sol.rotary_frequencies(2), 513)
    at = sample(tokens, 2 * dim, 1 << 26)
    kept, want = q[at], sol.rotary(q[at], None, table, at % 513, layout="interleaved")[0]
    say(f"  {tokens} tokens of a head of {dim} ({q.numel() * 2 / 2**30:.1f} GiB) in place")
    sol.rotary(q, None, table, layout="interleaved", q_out=q)
    assert torch.equal(q[at], want)
    # back again; every token's rotated pair keeps its length
    sol.rotary(q, None, table, layout="interleaved", inverse=True, q_out=q)
    assert torch.equal(q[at][..., 2:], kept[..., 2:])
    assert bool(((q[at] - kept)[..., :2].float().abs() <= 2.0 ** -6 * kept[..., :2].float().abs().amax(-1, True)).all())


def test_table_past_a_launch():
    """A pair a thread: 2^26 positions of 64 pairs are 2^32 threads."""
    rows = (1 << 26) + 5
    f = sol.rotary_frequencies(128).to(device())
    say(f"  table of {rows} positions ({rows * 128 * 4 / 2**30:.1f} GiB)")
    table = sol.rotary_table(f, rows)
    at = sample(rows, 512, 1 << 26)
    assert torch.equal(table[at], sol.rotary_table(f, at))
    # every angle's cosine and sine
    for i in range(0, rows, 1 << 24):
        t = table[i:i + (1 << 24)]
        assert float((t[:, :64].square() + t[:, 64:].square() - 1).abs().max()) < 2.0 ** -21


def test_rotary_past_a_launch_of_odd_waves():
    """11 waves a token: the workgroups of four that a launch ends with reach
    into the tokens after it, which must turn once all the same."""
    per_launch = 4 * ((1 << 24) - 1) // 11
    tokens, heads, dim = per_launch + 5, 22, 251
    assert per_launch * 11 % 4
    q = torch.empty((tokens, heads, dim), dtype=torch.bfloat16, device=device())
    q.normal_(generator=torch.Generator(device=device()).manual_seed(5))
    table = sol.rotary_table(sol.rotary_frequencies(2), 513)
    at = torch.cat((sample(tokens, 2 * heads * dim), torch.arange(per_launch - 5, tokens, device=device())))
    want = sol.rotary(q[at], None, table, at % 513, layout="interleaved")[0]
    say(f"  {tokens} tokens of {heads} heads of {dim} ({q.numel() * 2 / 2**30:.1f} GiB) in place")
    sol.rotary(q, None, table, layout="interleaved", q_out=q)
    assert torch.equal(q[at], want)


@pytest.mark.parametrize("kind", ["nvfp4", "mxfp8"])
def test_linear_past_a_launch(kind):
    """Tiles of 32 tokens in workgroups of 256 threads: 2^29 tokens are 2^32 threads."""
    M, N, K = (1 << 29) + 37, 3, 16 if kind == "nvfp4" else 32
    g = torch.Generator(device=device()).manual_seed(6)
    u8 = dict(dtype=torch.uint8, device=device())
    w = [torch.randint(256, (N, K // 2), generator=g, **u8),
         torch.randint(100, 140, (N, K // 32), generator=g, **u8) if kind == "mxfp8" else
         torch.randint(8, 120, (N, K // 16), generator=g, **u8)]
    if kind == "mxfp8":
        x = [torch.randint(0, 126, (M, K), generator=g, **u8), torch.randint(110, 130, (M, K // 32), generator=g, **u8)]
        call = sol.mxfp8_linear
    else:
        w.append(torch.ones(1, device=device()))
        x = [torch.empty((M, K), dtype=torch.bfloat16, device=device()).normal_(generator=g)]
        call = sol.nvfp4_weight_linear
    bias = torch.randn(N, generator=g, device=device()).bfloat16()
    say(f"  {kind} {M} x {N} x {K} ({x[0].numel() * x[0].element_size() / 2**30:.1f} GiB of activations)")
    out = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device=device())
    call(*x, *w, bias, out)
    at = torch.cat((sample(M, K * x[0].element_size(), 1 << 29), torch.arange((1 << 29) - 40, M, device=device())))
    assert torch.equal(out[at], call(*(t[at] for t in x), *w, bias))
    assert not bool(torch.isnan(out).any())
