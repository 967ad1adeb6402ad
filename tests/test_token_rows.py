"""The row arithmetic of the token cache (csrc/dc_token_cache.h, compiled for the host) against the definition: which rows hold what a token
sees, as sets, as runs and as steps of 64 rows; and the refusals of the entry points that need no device."""
import ctypes as C
import os
import random
import subprocess

import pytest

import paper_2609_35115_b200 as dc
from paper_2609_35115_b200 import binding

SRC = """
#include "dc_token_cache.h"
using namespace dc;
static CacheDims dims(int n_sink, int window, int ring) { return CacheDims{1, 1, 1, n_sink, window, ring}; }
extern "C" {
int row(int n_sink, int window, int ring, int pos) { return cache_row(dims(n_sink, window, ring), pos); }
unsigned long long mask(int n_sink, int window, int ring, int q_lo, int q_hi, int all, int r0) {
  const CacheDims d = dims(n_sink, window, ring);
  return mask64(all ? seen_by_all(d, q_lo, q_hi) : seen_by_any(d, q_lo, q_hi), n_sink, r0);
}
void runs(int n_sink, int window, int ring, int pos, int* out) {
  const RowRuns r = row_runs(dims(n_sink, window, ring), pos);
  out[0] = r.n_first; out[1] = r.lo_second; out[2] = r.n_second;
}
int steps(int n_sink, int window, int ring, int q_lo, int q_hi, int rank, int splits, int* out) {
  const CacheDims d = dims(n_sink, window, ring);
  StepList l;
  const int n = l.build(seen_by_any(d, q_lo, q_hi), n_sink, rank, splits);
  for (int j = 0; j < n; ++j) out[j] = l.tile(j);
  return n;
}
}
"""


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    d = tmp_path_factory.mktemp("token_rows")
    (d / "rows.cpp").write_text(SRC)
    pkg = os.path.dirname(dc.__file__)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-Wno-unknown-pragmas", "-I", os.path.join(pkg, "csrc"), "-I", os.path.join(os.path.dirname(pkg), "include"),
                    "-I", "/usr/local/cuda/include", "-o", str(d / "rows.so"), str(d / "rows.cpp")], check=True)
    lib = C.CDLL(str(d / "rows.so"))
    lib.mask.restype = C.c_ulonglong
    return lib


def held(n_sink, ring, last):
    """The position that every row holds after position `last` has been written (None: nothing)."""
    at = [None] * (n_sink + ring)
    for p in range(max(0, last + 1 - ring - n_sink - 1), last + 1):
        if p >= n_sink:
            at[n_sink + (p - n_sink) % ring] = p
    for p in range(min(n_sink, last + 1)):
        at[p] = p
    return at


def sees(q, p, n_sink, window):
    return p is not None and p <= q and (p < n_sink or p > q - window)


@pytest.mark.parametrize("seed", range(300))
def test_rows_of_a_window_are_those_of_the_definition(rows, seed):
    rng = random.Random(seed)
    n_sink, window, tokens = rng.choice([0, 1, 4, 63, 64, 70, 130]), rng.choice([1, 2, 31, 64, 100, 257]), rng.choice([1, 2, 7, 64, 90])
    ring = window + tokens - 1 + rng.choice([0, 1, 5, 64, 200])
    start = rng.choice([0, 1, n_sink, rng.randrange(3 * ring + n_sink + 2)])
    last = start + tokens - 1
    at = held(n_sink, ring, last)
    for p in range(start, last + 1):
        assert at[rows.row(n_sink, window, ring, p)] == p
    q_lo = start + rng.randrange(tokens)
    q_hi = rng.randrange(q_lo, last + 1)
    every = [[sees(q, p, n_sink, window) for p in at] for q in range(q_lo, q_hi + 1)]
    some, whole = [any(c) for c in zip(*every)], [all(c) for c in zip(*every)]
    n = n_sink + ring
    for want, flag in ((some, 0), (whole, 1)):
        for r0 in range(0, n + 64, 64):
            bits = rows.mask(n_sink, window, ring, q_lo, q_hi, flag, r0)
            assert [bool(bits >> i & 1) for i in range(64)] == [r0 + i < n and want[r0 + i] for i in range(64)], (r0, flag)
    # one token as two runs
    out = (C.c_int * 3)()
    rows.runs(n_sink, window, ring, q_lo, out)
    got = list(range(out[0])) + list(range(out[1], out[1] + out[2]))
    assert len(set(got)) == len(got) and sorted(got) == [r for r in range(n) if sees(q_lo, at[r], n_sink, window)]
    # steps: every tile that holds a seen row, once, over the CTAs of a cluster in order; none beyond the cache
    for splits in (1, 2, 8, 16):
        tiles, buf = [], (C.c_int * (n // 64 + 4))()
        for rank in range(splits):
            tiles += buf[:rows.steps(n_sink, window, ring, q_lo, q_hi, rank, splits, buf)]
        assert tiles == sorted({r // 64 for r in range(n) if some[r]})


# ---- refusals (no device is touched) -------------------------------------------------------------------------------------------

GOOD = dict(dtype=1, n_sessions=2, n_heads=8, n_kv_heads=2, head_dim=64, n_sink=4, window=32, ring_rows=40)


def open_raw(k=0x10000, v=0x20000, size=None, **kw):
    c = binding.dc_cache_config()
    c.size = C.sizeof(c) if size is None else size
    for name, x in {**GOOD, **kw}.items():
        setattr(c, name, x)
    h = C.c_void_p()
    st = dc.load_library().dc_cache_open(C.byref(c), k, v, C.byref(h))
    assert st != 0 and not h.value and dc.load_library().dc_last_error()
    return binding.STATUS[st]


@pytest.mark.parametrize("kw", [dict(dtype=0), dict(dtype=7), dict(n_sessions=0), dict(n_heads=7), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=130, n_kv_heads=2),
                                dict(n_heads=2048, n_kv_heads=2048), dict(head_dim=96), dict(head_dim=0), dict(n_sink=-1), dict(window=0), dict(window=41),
                                dict(ring_rows=2**31 - 1), dict(n_sessions=2**20, ring_rows=2**12), dict(size=8)])
def test_cache_configurations_outside_of_the_kernels_are_refused(kw):
    assert open_raw(**kw) == "DC_ERR_CONFIG"


def test_null_and_misaligned_caches_are_refused():
    assert open_raw(k=None) == "DC_ERR_ARG" and open_raw(v=None) == "DC_ERR_ARG"
    assert open_raw(k=0x10008) == "DC_ERR_ARG" and open_raw(v=0x20002) == "DC_ERR_ARG"
    assert open_raw(v=0x10000) == "DC_ERR_ARG"                                   # one memory for both
    assert open_raw(v=0x10000 + 2 * 2 * 44 * 64 * 2 - 16) == "DC_ERR_ARG"        # the last 16 bytes shared
    lib = dc.load_library()
    assert lib.dc_cache_open(None, 0x10000, 0x20000, None) == 1
    assert lib.dc_cache_close(None) == 1 and lib.dc_cache_check(None) == 1
    assert lib.dc_cache_append(None, None, None, None, 0, None, 0, None) == 1
    assert lib.dc_cache_attend(None, None, None, 0, 1.0, None, 0, None) == 1


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(n_rows=0), dict(n_rows=65536), dict(vocab=0), dict(vocab=262145, stride=262145), dict(stride=99), dict(logits=0x10004), dict(logits=None),
                                dict(u=None), dict(tokens=None), dict(size=4)])
def test_samples_outside_of_the_kernel_are_refused(kw):
    a = {**dict(dtype=0, n_rows=2, vocab=100, stride=100, logits=0x10000, u=0x20000, tokens=0x30000, size=C.sizeof(binding.dc_sample_rules)), **kw}
    r = binding.dc_sample_rules(a["size"])
    st = dc.load_library().dc_sample_tokens(a["logits"], a["dtype"], a["n_rows"], a["vocab"], a["stride"], C.byref(r), a["u"], a["tokens"], None, None)
    assert binding.STATUS[st] == "DC_ERR_ARG" and dc.load_library().dc_last_error()
