"""Launch forms of the operators over a token cache that only some sizes reach: single tokens over long windows (CTAs of 8 warps), rows dealt out over 4, 2 and 1
warps, tiles shared by 8 CTAs, both types at both head sizes, rounds that mix a prompt with single tokens, the last positions, a captured chunk."""
import math

import pytest
import torch

from tests import token_util as tu
from tests.test_gpu_token_cache import BF, HF, Case, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dc():
    import paper_2609_35115_b200 as dc
    dc.load_library()
    return dc


def attended(dc, **kw):
    c = Case(dc, **kw)
    q = c.normal(c.total, c.H, c.d)
    out = torch.full_like(q, 3.0)
    before = out.clone()
    c.cache.attend(q, c.batch, out=out)
    c.check_attend(q, out, before)
    assert torch.equal(c.cache.attend(q, c.batch, out=before.clone()), out)
    return c, q, out


# 256 units of 4 KB of rows or more, on no more than 148 CTAs
@pytest.mark.parametrize("H", [1, 7, 10, 17, 64])
@pytest.mark.parametrize("d,window", [(128, 4200), (64, 8300)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_single_tokens_over_long_windows(dc, dtype, d, window, H):
    attended(dc, dtype=dtype, d=d, H=H, Hkv=1, n_sink=5, window=window, new=(1, 1), start=(20000, window + 3), cu=False, seed=H)


@pytest.mark.parametrize("H,Hkv", [(2, 2), (12, 2), (24, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_in_fp16(dc, d, H, Hkv):
    attended(dc, dtype=HF, d=d, H=H, Hkv=Hkv, n_sink=3, window=300, new=(1, 1, 1), start=(900, 299, 2), cu=False, seed=H + d)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_shared_by_eight_ctas(dc, d, dtype):
    """16 to 31 steps of 64 rows, few tiles."""
    attended(dc, dtype=dtype, d=d, H=8, Hkv=2, n_sink=4, window=1200, new=(16, 9), start=(5000, 1190), seed=d)
    attended(dc, dtype=dtype, d=d, H=5, Hkv=1, n_sink=0, window=1500, new=(25,), start=(1480,), seed=d + 1)


@pytest.mark.parametrize("d,dtype", [(64, HF), (128, BF)])
def test_a_prompt_beside_single_tokens(dc, d, dtype):
    attended(dc, dtype=dtype, d=d, H=8, Hkv=2, n_sink=4, window=200, new=(333,) + (1,) * 12 + (0, 2), start=(40,) + tuple(37 * i for i in range(12)) + (5, 900), pad=3, seed=3)


@pytest.mark.parametrize("new,cu", [(1, False), (1, True), (40, True), (90, True)])
def test_the_last_positions(dc, new, cu):
    attended(dc, d=64, H=4, Hkv=2, n_sink=4, window=100, new=(new, new), start=(2 ** 31 - 2 - new, 2 ** 31 - 2 - new - 50), cu=cu, seed=4)


def test_a_captured_chunk_moves_on(dc):
    """The chunk's positions and boundaries are read when the graph runs."""
    c = Case(dc, new=(30, 11), start=(100, 400), d=64, H=8, Hkv=2, window=150, ring=300, seed=5)
    q = c.normal(c.total, 8, 64)
    start, cu, out, side = i32(c.start), i32(c.cu), torch.zeros_like(q), torch.cuda.Stream()
    batch = dc.TokenBatch(i32(c.order), start, cu, c.total, 40)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.cache.attend(q, batch, out=out)
    for new, at in (((30, 11), (100, 400)), ((1, 40), (777, 2)), ((41, 0), (5, 6))):      # (the last: more than max_tokens, left out)
        start.copy_(i32(at))
        cu.copy_(i32([0, new[0], sum(new)]))
        out.fill_(3)
        g.replay()
        torch.cuda.synchronize()
        c.new, c.start, c.cu, c.used = list(new), list(at), [0, new[0], sum(new)], sum(new)
        if new[0] > 40:
            assert (out == 3).all()
        else:
            c.check_attend(q, out, torch.full_like(out, 3.0))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (HF, 64), (HF, 128)])
@pytest.mark.parametrize("tokens", [5, 592, 593, 1300, 2500])
def test_append_of_many_tokens(dc, tokens, dtype, d, interleaved):
    """A row's pieces over 8, 4, 2 and 1 warps; two sequences and padding."""
    c = Case(dc, dtype=dtype, d=d, H=6, Hkv=2, n_sink=2, window=30, new=(tokens - 2, 2), start=(17, 0), pad=6, seed=tokens)
    x = (2 * torch.randn(c.total, 10 * d, generator=c.gen, device="cuda")).to(dtype)
    gains = [1 + 0.3 * torch.randn(d, generator=c.gen, device="cuda") for _ in range(2)]
    freq = torch.tensor([10000.0 ** (-2 * j / d) for j in range(d // 2)], device="cuda")
    q = torch.full((c.total, 6, d), 7.0, dtype=dtype, device="cuda")
    want_k, want_v = c.k.clone(), c.v.clone()
    c.cache.append(x, c.batch, dc.QKNorm(gains[0], gains[1], freq, interleaved=interleaved), q=q)
    for i in range(2):
        lo, hi, s = c.cu[i], c.cu[i + 1], c.order[i]
        rows, pos = [tu.row_of(p, c.n_sink, c.ring) for p in c.positions(i).tolist()], c.positions(i)
        y = x[lo:hi].double().view(hi - lo, 10, d)
        for part, gain, got in ((y[:, :6], gains[0], q[lo:hi]), (y[:, 6:8], gains[1], c.k[s][:, rows].transpose(0, 1))):
            want, size = tu.norm_rope(part.clone(), gain, pos, freq, 1e-6, interleaved)
            # half a step of the result, and 24 units of fp32 inside (sum of squares by a tree, root, gain, cosine and sine, two products and a sum)
            bound = tu.HALF[dtype] * want.abs() * 1.00001 + 24 * 2.0 ** -24 * size + 4 * math.pi * 2.0 ** -22 * size + tu.TINY[dtype]
            assert ((got.double() - want).abs() <= bound).all()
        want_k[s][:, rows] = c.k[s][:, rows]       # (checked above)
        want_v[s][:, rows] = x[lo:hi].view(hi - lo, 10, d)[:, 8:].transpose(0, 1)
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v) and (q[c.used:] == 7).all()
