"""The operators over a token cache (dc_cache_append, dc_cache_attend) against plain 64-bit forms: head layouts, types, lengths from one token
to prompts, rings that have wrapped, padded and ragged batches, strides, far positions, odd values in rows that are not seen; replays
of a captured step; and a run of the operators together."""
import math

import pytest
import torch

from tests import token_util as tu

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def dc():
    import paper_2609_35115_b200 as dc
    dc.load_library()
    return dc


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """Sessions with a history, and the tokens that a call brings."""

    def __init__(self, dc, dtype=BF, d=64, H=4, Hkv=2, n_sink=4, window=32, ring=None, new=(1,), start=(0,), pad=0, seed=0, pool=None, cu=True, fill="normal"):
        g = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.d, self.H, self.Hkv, self.n_sink, self.window = dtype, d, H, Hkv, n_sink, window
        self.ring = window + max(new) - 1 if ring is None else ring
        self.new, self.start, self.n = list(new), list(start), len(new)
        self.pool = self.n + 1 if pool is None else pool
        self.order = torch.randperm(self.pool, generator=g, device="cuda")[:self.n].tolist()
        self.rows = n_sink + self.ring
        shape = (self.pool, Hkv, self.rows, d)
        self.k, self.v = (self.normal(*shape) if fill == "normal" else torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(2))
        self.cu = [0]
        for t in self.new:
            self.cu.append(self.cu[-1] + t)
        self.used, self.total = self.cu[-1], self.cu[-1] + pad
        self.cache = dc.TokenCache(self.k, self.v, H, n_sink, window)
        single = not cu
        self.batch = dc.TokenBatch(i32(self.order), i32(self.start), None if single else i32(self.cu), self.total, max(max(self.new), 1))

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device="cuda").to(self.dtype)

    def positions(self, i):
        return torch.arange(self.start[i], self.start[i] + self.new[i], device="cuda")

    def seen_keys(self, i):
        """Positions that any token of sequence i may see, and their rows."""
        first, last = max(0, self.start[i] - self.window + 1), self.start[i] + self.new[i]
        keys = list(range(min(self.n_sink, first))) + list(range(first, last))
        return keys, [tu.row_of(p, self.n_sink, self.ring) for p in keys]

    def check_attend(self, q, out, before, scale=None):
        scale = self.d ** -0.5 if scale is None else scale
        for i in range(self.n):
            if not self.new[i]:
                continue
            keys, rows = self.seen_keys(i)
            s, lo, hi = self.order[i], self.cu[i], self.cu[i + 1]
            want, mag, worst = tu.attention(q[lo:hi].double(), self.k[s][:, rows].double(), self.v[s][:, rows].double(), torch.tensor(keys, device="cuda"), self.positions(i),
                                            self.n_sink, self.window, scale)
            got = out[lo:hi].double()
            bound = tu.attention_bound(want, mag, worst, len(keys), self.d, self.dtype, self.batch.c.max_tokens > 1)
            fine = torch.isfinite(want)
            assert torch.equal(torch.isnan(got), torch.isnan(want)), f"sequence {i}"
            assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
            over = ((got - want).abs() - bound)[fine]
            assert over.numel() == 0 or over.max() <= 0, f"sequence {i}: off by {float((got - want).abs()[fine].max())}, bound exceeded by {float(over.max())}"
        assert torch.equal(out[self.used:], before[self.used:])      # padding is left as it was
        self.cache.check()


# ---- append ------------------------------------------------------------------------------------------------------------------

APPEND = [
    dict(new=(1,), start=(0,), cu=False),
    dict(new=(1, 1, 1), start=(5, 0, 1000), cu=False, d=128, H=8, Hkv=1),
    dict(new=(1, 1), start=(2 ** 30, 2 ** 31 - 3), cu=False),                    # far positions
    dict(new=(3, 0, 7, 1), start=(0, 9, 33, 100), pad=5, d=128, H=6, Hkv=3, dtype=HF),
    dict(new=(20,), start=(50,), H=1, Hkv=1, n_sink=0, window=5),                # ring of 24, wrapped
    dict(new=(9, 2), start=(0, 2), H=28, Hkv=4, d=128, n_sink=3, window=1),
    dict(new=(2,) * 70, start=tuple(range(70)), H=2, Hkv=2, pad=1),              # more sequences than a warp has lanes
    dict(new=(5, 4), start=(0, 60), H=40, Hkv=8, d=64),
]


@pytest.mark.parametrize("rot", ["all", 32, 0])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append_against_64_bits(dc, case, interleaved, rot):
    c = Case(dc, seed=case, **APPEND[case])
    d, H, Hkv = c.d, c.H, c.Hkv
    rot = d if rot == "all" else rot
    width = (H + 2 * Hkv) * d
    wide = (2 * torch.randn(c.total, width + 24, generator=c.gen, device="cuda")).to(c.dtype)     # rows apart, as columns of a larger matrix
    qkv = wide[:, 8:8 + width]
    gains = [1 + 0.3 * torch.randn(d, generator=c.gen, device="cuda") for _ in range(2)]
    freq = torch.tensor([10000.0 ** (-2 * j / max(rot, 1)) for j in range(rot // 2)], device="cuda") if rot else None
    norm = dc.QKNorm(gains[0], gains[1], freq, eps=1e-5, interleaved=interleaved)
    q = torch.full((c.total, H, d), 7.0, dtype=c.dtype, device="cuda")
    k0, v0, q0 = c.k.clone(), c.v.clone(), q.clone()
    assert c.cache.append(qkv, c.batch, norm, q=q) is q
    want_k, want_v = k0.clone(), v0.clone()
    for i in range(c.n):
        lo, hi = c.cu[i], c.cu[i + 1]
        if hi == lo:
            continue
        x = qkv[lo:hi].double().view(hi - lo, H + 2 * Hkv, d)
        pos = c.positions(i)
        rows = [tu.row_of(p, c.n_sink, c.ring) for p in pos.tolist()]
        for part, gain, got in ((x[:, :H], gains[0], q[lo:hi]), (x[:, H:H + Hkv], gains[1], c.k[c.order[i]][:, rows].transpose(0, 1))):
            want, size = tu.norm_rope(part.clone(), gain, pos, freq, 1e-5, interleaved)
            # half a step of the result; fp32 inside: 64 or 128 squares summed by a tree with fused leaves (16 roundings, halved by the root), rsqrt, gain,
            # cos and sin (sincospi 2 units, the turn's own rounding to fp32 pi * 2^-24, the product in 64 bits 2^31 * 2^-53 turns), two products and a sum: 24 units of 2^-24
            bound = tu.HALF[c.dtype] * want.abs() * 1.00001 + 24 * 2.0 ** -24 * size + 2 * 2 * math.pi * 2.0 ** 31 * 2.0 ** -53 * size + tu.TINY[c.dtype]
            over = (got.double() - want).abs() - bound
            assert over.max() <= 0, f"sequence {i}: {float(over.max())}"
        want_k[c.order[i]][:, rows] = c.k[c.order[i]][:, rows]       # (checked above)
        want_v[c.order[i]][:, rows] = qkv[lo:hi].view(hi - lo, H + 2 * Hkv, d)[:, H + Hkv:].transpose(0, 1)
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v)     # rows of no token of the call are left as they were
    assert torch.equal(q[c.used:], q0[c.used:])


def test_append_in_place_and_odd_values(dc):
    c = Case(dc, new=(4, 3), start=(0, 30), d=128, H=4, Hkv=2)
    qkv = c.normal(c.total, 8 * 128)
    qkv[1, 5] = float("nan")                    # one head of one query
    qkv[2, 4 * 128 + 3] = float("inf")          # a key
    qkv[3, 7 * 128] = float("-inf")             # a value
    norm = dc.QKNorm(torch.ones(128, device="cuda"), torch.ones(128, device="cuda"), torch.full((64,), 0.5, device="cuda"))
    q = c.cache.append(qkv, c.batch, norm)
    k, v = c.k.clone(), c.v.clone()
    same = qkv.clone()
    got = c.cache.append(same, c.batch, norm, q=same[:, :4 * 128])
    assert torch.equal(got.reshape(7, 4, 128).nan_to_num(9), q.nan_to_num(9)) and torch.equal(same[:, 4 * 128:].nan_to_num(9), qkv[:, 4 * 128:].nan_to_num(9))
    assert torch.equal(c.k.nan_to_num(9), k.nan_to_num(9)) and torch.equal(c.v, v)
    bad = torch.isnan(q).flatten(1)
    assert bad[1, :128].all() and bad.sum() == 128          # a NaN stays in its head
    rows = [tu.row_of(p, c.n_sink, c.ring) for p in range(4)]
    assert v[c.order[0], 1, rows[3], 0] == float("-inf") and torch.isfinite(k[c.order[0]][:, rows[3]]).all()
    assert not torch.isfinite(k[c.order[0], 0, rows[2]]).all() and torch.isfinite(k[c.order[0], 1, rows[2]]).all()


# ---- attention -----------------------------------------------------------------------------------------------------------------

ATTEND = [
    # single tokens
    dict(new=(1,), start=(0,), cu=False),                                         # nothing but itself
    dict(new=(1, 1, 1, 1), start=(3, 4, 5, 300), cu=False),                       # around the first tokens, wrapped
    dict(new=(1, 1), start=(1000, 31), cu=False, d=128, H=8, Hkv=8, n_sink=0, window=1),
    dict(new=(1,), start=(5000,), cu=False, d=128, H=28, Hkv=4, n_sink=16, window=3000, ring=3001, dtype=HF),
    dict(new=(1,) * 5, start=(0, 77, 128, 513, 4000), cu=False, H=64, Hkv=1, n_sink=70, window=513),   # 64 heads of a group
    dict(new=(1,) * 40, start=tuple(7 * i for i in range(40)), cu=False, H=8, Hkv=8, window=100),
    dict(new=(1, 0, 1), start=(90, 5, 20), pad=3, H=5, Hkv=1, d=128),             # a sequence without tokens, padding
    dict(new=(1,), start=(63,), cu=False, n_sink=64, window=64, ring=64),
    # chunks
    dict(new=(2,), start=(0,)),
    dict(new=(3, 17, 0, 1), start=(0, 40, 9, 100), pad=7, d=128, H=6, Hkv=3),
    dict(new=(50, 23), start=(700, 11), d=64, H=8, Hkv=8, n_sink=30, window=256, ring=320),
    dict(new=(64,), start=(64,), d=128, H=4, Hkv=4, n_sink=64, window=64, ring=128),
    dict(new=(40, 33), start=(1000, 2000), d=128, H=7, Hkv=1, n_sink=1, window=33, dtype=HF),
    dict(new=(30,), start=(333,), d=64, H=64, Hkv=1, n_sink=5, window=90),
    dict(new=(90,), start=(0,), d=128, H=2, Hkv=1, n_sink=3, window=1, ring=90),   # a window of the token alone
    dict(new=(12, 1, 5), start=(4000, 1, 3000), d=128, H=8, Hkv=2, n_sink=0, window=2500),   # few tiles, long rows: split over clusters
    dict(new=(16,), start=(200,), d=64, H=4, Hkv=2, n_sink=130, window=700),
    # prompts
    dict(new=(700,), start=(0,), d=128, H=4, Hkv=2, n_sink=4, window=128),
    dict(new=(515, 300), start=(100, 0), d=64, H=8, Hkv=2, n_sink=0, window=2000, dtype=HF),
    dict(new=(1100,), start=(777,), d=128, H=2, Hkv=2, n_sink=70, window=600, ring=1900),
]


@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_against_64_bits(dc, case):
    c = Case(dc, seed=100 + case, **ATTEND[case])
    q = c.normal(c.total, c.H, c.d)
    out = torch.full_like(q, 3.0)
    before = out.clone()
    k, v = c.k.clone(), c.v.clone()
    assert c.cache.attend(q, c.batch, out=out) is out
    c.check_attend(q, out, before)
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    assert torch.equal(c.cache.attend(q, c.batch, out=before.clone()), out)       # the same bytes again


@pytest.mark.parametrize("case", [1, 4, 9, 12, 15, 17])
def test_attention_with_strides_scale_and_sharp_scores(dc, case):
    c = Case(dc, seed=200 + case, **ATTEND[case])
    wide = (4 * torch.randn(c.total, c.H * c.d + 40, generator=c.gen, device="cuda")).to(c.dtype)
    c.k *= 3
    q = wide[:, 16:16 + c.H * c.d]
    holder = torch.full((c.total, c.H * c.d + 8), 3.0, dtype=c.dtype, device="cuda")
    out, before = holder[:, :c.H * c.d], holder.clone()
    c.cache.attend(q, c.batch, out=out, scale=0.25)
    c.check_attend(q.unflatten(1, (c.H, c.d)), out.unflatten(1, (c.H, c.d)), before[:, :c.H * c.d].unflatten(1, (c.H, c.d)), scale=0.25)
    assert torch.equal(holder[:, c.H * c.d:], before[:, c.H * c.d:])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), "lowest"])
@pytest.mark.parametrize("case", [0, 1, 4, 6, 8, 9, 10, 12, 14, 15, 17])
def test_rows_that_are_not_seen_may_hold_anything(dc, case, value):
    """Everything but the seen rows is odd: rows not written yet, evicted ones, other sessions."""
    c0 = Case(dc, seed=300 + case, **ATTEND[case])
    fill = torch.finfo(c0.dtype).min if value == "lowest" else value
    c = Case(dc, seed=300 + case, fill=fill, **ATTEND[case])
    for i in range(c.n):
        _, rows = c.seen_keys(i)
        if c.new[i]:
            c.k[c.order[i]][:, rows], c.v[c.order[i]][:, rows] = (c.normal(c.Hkv, len(rows), c.d) for _ in range(2))
    q = c.normal(c.total, c.H, c.d)
    out = torch.zeros_like(q)
    c.cache.attend(q, c.batch, out=out)
    assert torch.isfinite(out[:c.used]).all()
    c.check_attend(q, out, torch.zeros_like(q))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("case", [9, 10, 12, 15, 17])
def test_an_odd_value_reaches_the_tokens_that_see_it_and_no_other(dc, case, value):
    c = Case(dc, seed=400 + case, **ATTEND[case])
    i = max(range(c.n), key=lambda j: c.new[j])
    s, p = c.order[i], c.start[i] + c.new[i] // 2                       # a token in the middle of the chunk: later ones see it
    c.v[s][0, tu.row_of(p, c.n_sink, c.ring), 5] = value
    if c.start[i] > c.window:                                           # and the oldest one that the first token sees
        c.v[s][-1, tu.row_of(max(c.n_sink, c.start[i] - c.window + 1), c.n_sink, c.ring), 6] = value
    q = c.normal(c.total, c.H, c.d)
    out = torch.zeros_like(q)
    c.cache.attend(q, c.batch, out=out)
    c.check_attend(q, out, torch.zeros_like(q))
    lo, hi = c.cu[i], c.cu[i + 1]
    assert torch.isfinite(out[lo:lo + c.new[i] // 2, 0, 5]).all() and not torch.isfinite(out[lo + c.new[i] // 2, 0, 5])
    # a key: a NaN score is the token's own affair too
    c.k[s][0, tu.row_of(p, c.n_sink, c.ring), 9] = float("nan")
    c.cache.attend(q, c.batch, out=out)
    G = c.H // c.Hkv
    assert torch.isnan(out[lo + c.new[i] // 2, :G]).all() and not torch.isnan(out[lo:lo + c.new[i] // 2, 0, 0]).any()
    c.cache.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_sink,ring,T", [(0, 1, 1), (1, 1, 1), (0, 2, 2), (2, 3, 3), (0, 63, 40), (5, 59, 59)])
def test_the_smallest_caches(dc, n_sink, ring, T, d):
    """Fewer rows than a box of the copies, a window that is as long as the ring lets it."""
    c = Case(dc, new=(T,), start=(7 * ring,), d=d, H=3, Hkv=1, n_sink=n_sink, window=ring - T + 1, ring=ring, pool=1, seed=ring)
    q = c.normal(c.total, 3, d)
    out = torch.zeros_like(q)
    c.cache.attend(q, c.batch, out=out)
    c.check_attend(q, out, torch.zeros_like(q))


# ---- batches that do not fit, refusals ---------------------------------------------------------------------------------------------


@pytest.mark.parametrize("tokens", [1, 6])
def test_sequences_with_values_that_do_not_fit_are_left_out(dc, tokens):
    c = Case(dc, new=(tokens,) * 8, start=(10,) * 8, d=64, H=4, Hkv=2, pad=2)
    n, big = 8, 2 ** 31 - 1
    sessions, start, cu = c.order[:], c.start[:], c.cu[:]
    sessions[0], sessions[1] = c.pool, -1
    start[2], start[3] = -1, big
    start[4] = -2 ** 31
    cu[7] = c.total + 5                      # sequence 6 ends behind the matrices, sequence 7 begins there
    batch = dc.TokenBatch(i32(sessions), i32(start), i32(cu), c.total, tokens)
    q = c.normal(c.total, c.H, c.d)
    out = torch.full_like(q, 3.0)
    c.cache.attend(q, batch, out=out)
    norm = dc.QKNorm(torch.ones(64, device="cuda"), torch.ones(64, device="cuda"))
    qkv, y = c.normal(c.total, 8 * 64), torch.full_like(q, 3.0)
    k0 = c.k.clone()
    c.cache.append(qkv, batch, norm, q=y)
    for t in (out, y):
        assert (t[:5 * tokens] == 3).all() and (t[6 * tokens:] == 3).all() and (t[5 * tokens:6 * tokens] != 3).any()
    changed = (c.k != k0).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [c.order[5]]
    # more tokens than max_tokens says
    if tokens > 1:
        short = dc.TokenBatch(i32(c.order), i32(c.start), i32(c.cu), c.total, tokens - 1)
        out.fill_(3)
        c.cache.attend(q, short, out=out)
        assert (out == 3).all()
    c.cache.check()


def test_refusals(dc):
    c = Case(dc, new=(3, 2), start=(0, 0), d=64, H=4, Hkv=2, window=8, ring=10)
    q, norm = c.normal(5, 4, 64), dc.QKNorm(torch.ones(64, device="cuda"), torch.ones(64, device="cuda"))

    def status(call):
        with pytest.raises(dc.DCError) as e:
            call()
        return dc.STATUS[e.value.status]

    assert status(lambda: c.cache.attend(q, dc.TokenBatch(i32([0, 1]), i32([0, 0]), i32([0, 3, 5]), 5, 4))) == "DC_ERR_FRAMES"     # the ring takes 3
    assert status(lambda: c.cache.attend(q[:2], dc.TokenBatch(i32([0, 1]), i32([0, 0]), None, 2, 2))) == "DC_ERR_ARG"
    assert status(lambda: c.cache.attend(q[:5], dc.TokenBatch(i32([0, 1]), i32([0, 0]), None, 5, 1))) == "DC_ERR_ARG"
    assert status(lambda: c.cache.attend(q, dc.TokenBatch(i32([0, 1]), i32([0, 0]), i32([0, 3, 5]), 5, 0))) == "DC_ERR_ARG"
    assert status(lambda: c.cache.attend(q[:4], dc.TokenBatch(None, i32([0] * 4)))) == "DC_ERR_ARG"                               # 3 sessions
    for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        assert status(lambda: c.cache.attend(q, c.batch, scale=scale)) == "DC_ERR_ARG"
    wide = torch.zeros(5, 4 * 64 + 4, dtype=BF, device="cuda")
    assert status(lambda: c.cache.attend(wide[:, :256], c.batch)) == "DC_ERR_ARG"                 # rows 520 bytes apart
    flat = torch.zeros(5 * 256 + 8, dtype=BF, device="cuda")
    assert status(lambda: c.cache.attend(flat[1:1281].view(5, 4, 64), c.batch)) == "DC_ERR_ARG"   # misaligned
    qkv = c.normal(5, 8 * 64)
    assert status(lambda: c.cache.append(qkv, c.batch, dc.QKNorm(torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(4, device="cuda")))) == "DC_ERR_ARG"
    assert status(lambda: c.cache.append(qkv, c.batch, dc.QKNorm(torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(40, device="cuda")))) == "DC_ERR_ARG"
    assert status(lambda: c.cache.append(qkv, c.batch, dc.QKNorm(torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), eps=-1.0))) == "DC_ERR_ARG"
    for call in (lambda: c.cache.attend(q.half(), c.batch), lambda: c.cache.attend(q[:4], c.batch), lambda: c.cache.attend(q.cpu(), c.batch),
                 lambda: c.cache.attend(q.transpose(1, 2), c.batch), lambda: c.cache.append(q, c.batch, norm),
                 lambda: dc.TokenBatch(i32([0, 1]), i32([0, 0]).long()), lambda: dc.TokenBatch(i32([0]), i32([0, 0])), lambda: dc.TokenBatch(None, i32([0, 0]), i32([0, 1]), 1, 1), lambda: dc.TokenBatch(None, i32([0, 0]), i32([0, 1, 2]), 2), lambda: dc.TokenBatch(None, i32([0, 0]), i32([0, 1, 2]), max_tokens=1),
                 lambda: dc.TokenCache(c.k[:, :, ::2], c.v[:, :, ::2], 4), lambda: dc.TokenCache(c.k, c.v[:2], 4), lambda: dc.QKNorm(torch.ones(64), torch.ones(64))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        dc.TokenCache(c.k.double(), c.v.double(), 4)
    # nothing of this has left the device in an error state
    out = torch.zeros_like(q)
    c.cache.attend(q, c.batch, out=out)
    c.check_attend(q, out, torch.zeros_like(q))


# ---- a step as it is used ------------------------------------------------------------------------------------------------------------


def test_a_prompt_and_steps_agree_with_one_long_prompt(dc):
    """A prompt, then single tokens, against the same positions as one prompt: every token sees the same rows, whatever call brought it."""
    T, n0, d, H, Hkv = 150, 61, 128, 8, 2
    one = Case(dc, new=(T,), start=(0,), d=d, H=H, Hkv=Hkv, n_sink=3, window=40, seed=5)
    qkv = one.normal(T, (H + 2 * Hkv) * d)
    norm = dc.QKNorm(1 + 0.1 * torch.randn(d, generator=one.gen, device="cuda"), torch.ones(d, device="cuda"), torch.tensor([100.0 ** (-j / 64) for j in range(64)], device="cuda"))
    q = one.cache.append(qkv, one.batch, norm)
    want = one.cache.attend(q, one.batch)
    one.check_attend(q, want, want)

    two = Case(dc, new=(n0,), start=(0,), d=d, H=H, Hkv=Hkv, n_sink=3, window=40, ring=100, seed=6, fill=float("nan"))
    got = [two.cache.attend(two.cache.append(qkv[:n0], two.batch, norm), two.batch)]
    # the single step as a captured graph: what moves on is the position, in place
    start = i32([n0])
    batch, x, out = dc.TokenBatch(i32(two.order), start), torch.empty_like(qkv[:1]), torch.empty(1, H, d, dtype=BF, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = two.cache.append(x.copy_(qkv[n0:n0 + 1]), batch, norm)
        two.cache.attend(y, batch, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        two.cache.append(x, batch, norm, q=y)
        two.cache.attend(y, batch, out=out)
        start += 1
    for t in range(n0, T):
        x.copy_(qkv[t:t + 1])
        graph.replay()
        got.append(out.clone())
    got = torch.cat(got).double()
    # both are within their bound of the exact values of (rounded) q, k, v, which are the same bytes
    k = torch.stack([one.k[one.order[0]][:, tu.row_of(p, 3, one.ring)] for p in range(T)], 1).double() if one.ring >= T - 3 else None
    if k is not None:
        v = torch.stack([one.v[one.order[0]][:, tu.row_of(p, 3, one.ring)] for p in range(T)], 1).double()
        exact, mag, worst = tu.attention(q.double(), k, v, torch.arange(T, device="cuda"), torch.arange(T, device="cuda"), 3, 40, d ** -0.5)
        assert ((got - exact).abs() <= tu.attention_bound(exact, mag, worst, 43, d, BF, True)).all()
    two.cache.check()


def test_two_streams_and_two_caches_at_once(dc):
    """Calls on two streams, over caches and batches of their own, give what they give one after the other."""
    cs = [Case(dc, new=(1,) * 6, start=(500,) * 6, d=128, H=8, Hkv=2, window=400, cu=False, seed=7), Case(dc, new=(30,) * 3, start=(90,) * 3, d=64, H=8, Hkv=8, window=90, seed=8)]
    qs = [c.normal(c.total, c.H, c.d) for c in cs]
    want = [c.cache.attend(q, c.batch) for c, q in zip(cs, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    outs = [[torch.empty_like(q) for _ in range(20)] for q in qs]
    for r in range(20):
        for c, q, s, o in zip(cs, qs, streams, outs):
            c.cache.attend(q, c.batch, out=o[r], stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, x) for x in o)


def test_a_cache_with_offsets_behind_32_bits(dc):
    """A pool whose last session lies behind 2^32 values."""
    pool, rows, Hkv, d = 9, 524288 + 64, 8, 128          # 4.8e9 values of keys
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("not enough free memory")
    k, v = (torch.zeros(pool, Hkv, rows, d, dtype=BF, device="cuda") for _ in range(2))
    cache = dc.TokenCache(k, v, 8, 4, 50)
    g = torch.Generator(device="cuda").manual_seed(1)
    norm = dc.QKNorm(torch.ones(d, device="cuda"), torch.ones(d, device="cuda"))
    for T, start in ((20, rows - 30), (1, rows - 10)):
        batch = dc.TokenBatch(i32([pool - 1]), i32([start]), i32([0, T]), T, T)
        qkv = torch.randn(T, 24 * d, generator=g, device="cuda").to(BF)
        out = cache.attend(cache.append(qkv, batch, norm), batch)
        first = max(0, start - 49)
        keys = list(range(4)) + list(range(first, start + T))
        r = [tu.row_of(p, 4, rows - 4) for p in keys]
        q = tu.norm_rope(qkv.double().view(T, 24, d)[:, :8], torch.ones(d, device="cuda"), None, None, 1e-6, False)[0].to(BF).double()
        want, mag, worst = tu.attention(q, k[pool - 1][:, r].double(), v[pool - 1][:, r].double(), torch.tensor(keys, device="cuda"), torch.arange(start, start + T, device="cuda"),
                                        4, 50, d ** -0.5)
        bound = tu.attention_bound(want, mag, worst, len(keys), d, BF, T > 1) + 2 * worst * tu.HALF[BF] * mag      # (q is rounded apart: a score may be half a step of q off)
        assert ((out.double() - want).abs() <= bound).all()
        assert torch.equal(v[pool - 1][:, r[-1]], qkv.view(T, 24, d)[-1, 16:])
    cache.close()


def test_caches_come_and_go_while_a_step_is_captured(dc):
    """Opening, using and closing a cache inside of a capture: nothing of it touches the device outside of the stream."""
    c = Case(dc, new=(1, 1), start=(40, 3), d=64, H=4, Hkv=2, cu=False, seed=9)
    q = c.normal(2, 4, 64)
    want = c.cache.attend(q, c.batch)
    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        again = dc.TokenCache(c.k, c.v, 4, c.n_sink, c.window)
        again.attend(q, c.batch, out=out)
        again.close()
        del again
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_two_graphs_over_one_cache_at_once(dc):
    """Two captured steps of different sessions of one cache, replayed on two streams: calls have no memory of their own to share."""
    c = Case(dc, new=(1,) * 8, start=(900,) * 8, d=128, H=8, Hkv=2, window=600, cu=False, seed=10)
    parts = [dc.TokenBatch(i32(c.order[i:i + 4]), i32([900] * 4)) for i in (0, 4)]
    q = [c.normal(4, 8, 128) for _ in parts]
    want = [c.cache.attend(x, b) for x, b in zip(q, parts)]
    torch.cuda.synchronize()
    streams, graphs, outs = [torch.cuda.Stream() for _ in parts], [], []
    for x, b, s in zip(q, parts, streams):
        o, g = torch.zeros_like(x), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            for _ in range(10):
                c.cache.attend(x, b, out=o)
        graphs.append(g)
        outs.append(o)
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_chunks_beside_the_flow_decoder(dc):
    """A chunk's attention (tensor memory, clusters) on one stream, the flow decoder on another."""
    import numpy as np
    import dc_workloads as wl
    cfg = wl.tiny_flow(name="beside", n_chunks=3, seed=3)
    w = wl.make_workload(cfg)
    m = dc.Model(cfg, w.weights)
    st = m.open_stream()
    feats = torch.from_numpy(np.ascontiguousarray(w.streams[0].feats[:cfg.f_chunk])).cuda()
    c = Case(dc, new=(40,) * 4, start=(300,) * 4, d=64, H=16, Hkv=2, window=300, seed=11)
    q = c.normal(c.total, 16, 64)
    want = c.cache.attend(q, c.batch)
    first = st.decode_chunk(feats).clone()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [torch.empty_like(q) for _ in range(30)]
    got = []
    for o in outs:
        with torch.cuda.stream(b):
            st.reset(stream=b)
            got.append(st.decode_chunk(feats, out=torch.empty(feats.shape[0] * m.out_per_frame, device="cuda"), stream=b))
        c.cache.attend(q, c.batch, out=o, stream=a)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs) and all(torch.equal(x.reshape(-1), first.reshape(-1)) for x in got)
    assert m.counters()[4] == 0
    c.cache.check()
    st.close()
    m.destroy()
