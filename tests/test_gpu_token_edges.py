"""The ends of the token operators' ranges: the largest sums, scores and values, results on other streams, and the launch forms that few calls reach."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import pick
from tests.test_gpu_token_cache import BF, HF, Case, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dc():
    import paper_2609_35115_b200 as dc
    dc.load_library()
    return dc


# ---- sampling ------------------------------------------------------------------------------------------------------------------


def test_masses_of_flat_rows_of_the_largest_vocabulary(dc):
    """Rows that begin off a 16-byte border: a thread adds up to 260 weights close to one, whose sum passes 2^53 units of 2^-45.  The last tokens weigh nothing, so
    that the last kept one lies at the end of the part of a warp whose threads have that many."""
    n, vocab, kept = 150, 262144, 262144 - 6276
    rng = np.random.default_rng(21)
    g = torch.Generator(device="cuda").manual_seed(21)
    l = torch.randn(n, vocab + 1, generator=g, device="cuda")[:, :vocab]
    l[:, kept:] = -torch.inf
    u = torch.tensor(np.where(np.arange(n) % 3 == 0, rng.random(n), 1.0), dtype=torch.float32, device="cuda")
    T = torch.full((n,), 1e3, device="cuda")
    tokens, probs = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), 9.0, device="cuda")
    dc.sample_tokens(l, u, temperature=T, tokens=tokens, probs=probs)
    got, share = tokens.tolist(), probs.tolist()
    for r in range(n):
        if r % 3:      # u = 1: the last kept token, whatever the others weigh
            assert got[r] == kept - 1 and 0 < share[r] < 1e-5, r
        else:
            want, p = pick(l[r].double().cpu().numpy(), float(u[r]), 1e3)
            assert got[r] == want and abs(share[r] - p) <= 2.0 ** -24 * p * 1.001, r


# ---- attention: scores and values at the ends of their range ----------------------------------------------------------------------


@pytest.mark.parametrize("scale", [2.0 ** 20, 2.0 ** 25, 1e10, 2.0 ** 33, 1e30])
@pytest.mark.parametrize("new", [1, 40, 300])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (HF, 128)])
def test_scores_far_beyond_fp32s_whole_numbers(dc, dtype, d, new, scale):
    """One value of each key counts, and no two keys have the same (in the types' 8 bits, exactly): every other score lies far below the largest one a token sees,
    so its output is that key's row of V, bit for bit."""
    window = 100
    c = Case(dc, new=(new,), start=(150,), d=d, H=4, Hkv=2, n_sink=3, window=window, dtype=dtype, seed=31, cu=new > 1)
    g = torch.Generator(device="cuda").manual_seed(32)
    keys, rows = c.seen_keys(0)
    value = 1.0 + torch.randperm(128, generator=g, device="cuda")[torch.arange(len(keys), device="cuda") % 128].double() / 128      # distinct in any window and its first tokens
    s = c.order[0]
    c.k.zero_()
    c.k[s][:, rows, 0] = value.to(dtype)
    c.k[s][:, rows[:3], 0] = 0.5                        # (the first tokens, once they are out of the window)
    q = torch.zeros(c.total, 4, d, dtype=dtype, device="cuda")
    q[:, :, 0] = 1.0
    out = c.cache.attend(q, c.batch, scale=scale)
    key = torch.tensor(keys, device="cuda")
    for t, at in enumerate(c.positions(0).tolist()):
        seen = (key <= at) & (key > at - window)
        best = torch.where(seen, value, -1.0).argmax()
        want = c.v[s][:, rows[int(best)]].repeat_interleave(2, 0)
        assert torch.equal(out[t], want), (t, at)
    c.cache.check()


@pytest.mark.parametrize("new", [1, 40, 700])
def test_values_at_fp16s_largest_stay_finite(dc, new):
    """Rows of V of the type's largest value: a weighted mean of them is that value, never above."""
    c = Case(dc, new=(new,), start=(900,), d=64, H=4, Hkv=2, window=512, dtype=HF, seed=41, cu=new > 1)
    top = torch.finfo(HF).max
    sign = torch.where(torch.arange(64, device="cuda") % 2 == 0, 1.0, -1.0)
    c.v.copy_((top * sign).to(HF).expand_as(c.v))
    q = (3 * torch.randn(c.total, 4, 64, generator=c.gen, device="cuda")).to(HF)
    out = c.cache.attend(q, c.batch)
    assert torch.isfinite(out).all()
    c.check_attend(q, out, out)
    # an infinity or a NaN that tokens see stays visible, in its column alone
    keys, rows = c.seen_keys(0)
    c.v[c.order[0], 0, rows[0], 0], c.v[c.order[0], 1, rows[1], 1] = float("inf"), float("nan")      # (first tokens)
    q.zero_()
    c.cache.attend(q, c.batch, out=out)
    assert not torch.isfinite(out[:, :2, 0]).any() and torch.isnan(out[:, 2:, 1]).all() and torch.isfinite(out[:, :2, 1:]).all()
    c.cache.check()


# ---- results that a call allocates itself ----------------------------------------------------------------------------------------------


def behind_queued_work(like, call):
    """What `call` returns while the current stream still holds queued writes to memory that it has given back."""
    torch.cuda.synchronize()
    held = [torch.empty_like(like) for _ in range(64)]
    torch.cuda._sleep(200_000_000)
    for t in held:
        t.fill_(7)
    del held, t
    got = call()
    torch.cuda.synchronize()
    return got


def test_results_on_another_stream_lie_in_memory_of_that_stream(dc):
    side = torch.cuda.Stream()
    c = Case(dc, new=(1,) * 6, start=(50,) * 6, d=128, H=8, Hkv=2, window=40, cu=False, seed=51)
    q = c.normal(6, 8, 128)
    want = c.cache.attend(q, c.batch)
    assert torch.equal(behind_queued_work(want, lambda: c.cache.attend(q, c.batch, stream=side)), want)
    assert torch.equal(behind_queued_work(want, lambda: c.cache.attend(q, c.batch, stream=side.cuda_stream)), want)      # a plain handle
    qkv, norm = c.normal(6, 12 * 128), dc.QKNorm(torch.ones(128, device="cuda"), torch.ones(128, device="cuda"))
    want = c.cache.append(qkv, c.batch, norm)
    assert torch.equal(behind_queued_work(want, lambda: c.cache.append(qkv, c.batch, norm, stream=side)), want)
    logits, u = torch.randn(6, 1000, device="cuda"), torch.full((6,), 0.5, device="cuda")
    want = dc.sample_tokens(logits, u)
    assert torch.equal(behind_queued_work(want, lambda: dc.sample_tokens(logits, u, stream=side)), want)
    assert torch.equal(dc.sample_tokens(logits, u, stream=0), want)
    c.cache.check()


def test_decoded_audio_on_another_stream_lies_in_memory_of_that_stream(dc):
    import dc_workloads as wl
    cfg = wl.tiny_flow(name="elsewhere", n_chunks=3, seed=5)
    w = wl.make_workload(cfg)
    m, side = dc.Model(cfg, w.weights, max_batch=cfg.n_steps), torch.cuda.Stream()
    st = m.open_stream()
    feats = torch.from_numpy(np.ascontiguousarray(w.streams[0].feats[:2 * cfg.f_chunk])).cuda()
    for call in (lambda s: st.decode_chunk(feats[:cfg.f_chunk], stream=s), lambda s: st.decode_wavefront(feats, stream=s), lambda s: dc.decode_wavefront_batch(m, [st], [feats], stream=s)[0]):
        st.reset()
        want = call(None)
        torch.cuda.synchronize()
        st.reset()
        assert torch.equal(behind_queued_work(want, lambda: call(side)), want)
    st.close()
    m.destroy()


def test_rules_that_are_no_numbers_or_out_of_range(dc):
    """A NaN as top_p or min_p rules nothing out; min_p above 1 is as 1: the logits that tie with the largest."""
    g = torch.Generator(device="cuda").manual_seed(61)
    for vocab in (50, 9000):
        l, u = torch.round(torch.randn(40, vocab, generator=g, device="cuda") * 2), torch.rand(40, generator=g, device="cuda")
        every = lambda x: torch.full((40,), x, device="cuda")
        free = dc.sample_tokens(l, u)
        assert torch.equal(dc.sample_tokens(l, u, top_p=every(float("nan"))), free) and torch.equal(dc.sample_tokens(l, u, min_p=every(float("nan"))), free)
        best = dc.sample_tokens(l, u, min_p=every(1.0))
        assert torch.equal(dc.sample_tokens(l, u, min_p=every(7.0)), best)
        assert torch.equal(l.gather(1, best.long()[:, None])[:, 0], l.amax(1))
