"""Host-side tests of the prefix-cache operators: the oracle's own pins, sizes,
and refusals.  No GPU needed: everything here returns before work is enqueued."""
import ctypes as C
import dataclasses
import os
import re

import numpy as np
import pytest

from oracle import kv as okv
from paper_2607_01088_amd import rosa
from synthetic import PI0_SHAPE, TINY_SHAPE
from tests.helpers import ROOT

A = 0x10000      # device addresses that host checks never dereference


def test_library_exports_every_function_of_the_header():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rosa_kv.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rosa_[a-z0-9_]+)\s*\(", src)))
    assert len(names) >= 10
    for n in names:
        assert hasattr(rosa.load(), n), n


# ---------------------------------------------------------------- the oracle

def test_oracle_rounds_to_the_nearest_code_and_ties_to_even():
    x = np.zeros(32)
    x[:15] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.26, 0.74, 2.51, -0.25, -0.75, -5.01, 0.24]
    c, s = okv.quantize(x[None])
    assert s[0, 0] == 127
    v = okv.expand(c, s)[0]
    assert list(v[:15]) == [6, 0, 1, 1, 2, 2, 4, 4, 0.5, 0.5, 3, 0, -1, -6, 0]


def test_oracle_scale_is_the_least_power_of_two_with_seven_times_it_at_or_above_the_maximum():
    for e in range(-120, 120, 7):
        for a, want in [(7 * 2.0 ** e, e), (np.nextafter(7 * 2.0 ** e, np.inf), e + 1), (3.6 * 2.0 ** e, e), (3.5 * 2.0 ** e, e - 1)]:
            x = np.zeros((1, 32))
            x[0, 5] = -a
            assert okv.block_exponents(x)[0, 0] == want, (e, a)
    for a, want in [(0.0, -125), (1e-300, -125), (3.3e38, 125), (np.inf, 128), (np.nan, 128)]:
        assert okv.block_exponents(np.full((1, 32), a))[0, 0] == want


def test_oracle_expand_brute_force():
    rng = np.random.default_rng(0)
    c, s = rng.integers(0, 256, (3, 16), dtype=np.uint8), rng.integers(2, 253, (3, 1), dtype=np.uint8)
    v = okv.expand(c, s)
    for r in range(3):
        for i in range(32):
            n = (c[r, i // 2] >> (4 * (i % 2))) & 15
            ex, man = (n >> 1) & 3, n & 1
            mag = man * 0.5 if ex == 0 else (1 + man / 2) * 2.0 ** (ex - 1)
            assert v[r, i] == (-1 if n & 8 else 1) * mag * 2.0 ** (int(s[r, 0]) - 127)


def test_oracle_attention_agrees_with_scalar_loops_and_masses_sum_to_the_rows():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    o, lse, w = okv.attend(q, k, v)
    for t in range(3):
        for g in range(4):
            s = [sum(q[t, g, i] * k[j, g // 2, i] for i in range(8)) / np.sqrt(8) for j in range(5)]
            l = np.log(sum(np.exp(x) for x in s))
            assert abs(l - lse[t, g]) < 1e-12
            for i in range(8):
                assert abs(sum(np.exp(s[j] - l) * v[j, g // 2, i] for j in range(5)) - o[t, g, i]) < 1e-12
    np.testing.assert_allclose(okv.masses(w, 2, 5).sum(-1), [6, 6], rtol=1e-12)


def test_oracle_keeps_protected_then_largest_ties_to_the_lowest_index_nan_last():
    m = np.array([0, 5, 1, 5, np.nan, 5, -np.inf, 0], np.float32)
    assert list(okv.keep_tokens(m, 4, 1, 1)) == [0, 1, 3, 7]
    assert list(okv.keep_tokens(m, 3, 0, 0)) == [1, 3, 5]
    assert list(okv.keep_tokens(m, 7, 0, 0)) == [0, 1, 2, 3, 5, 6, 7]
    assert list(okv.keep_tokens(m, 2, 1, 1)) == [0, 7]


# ---------------------------------------------------------------- sizes and refusals

def test_bytes():
    assert rosa.kv_bytes(PI0_SHAPE, "bf16", rosa.ROSA_KV_MODEL, 100) == 18 * 100 * 256 * 2
    assert rosa.kv_bytes(PI0_SHAPE, "bf16", rosa.ROSA_KV_FP4, 100) == 18 * 100 * (128 + 8)
    assert rosa.kv_bytes(PI0_SHAPE, "fp32", rosa.ROSA_KV_MODEL, 0) == 0
    assert rosa.kv_bytes(PI0_SHAPE, "bf16", rosa.ROSA_KV_FP4, 2 ** 31 - 1) == 18 * (2 ** 31 - 1) * 136
    for fmt, P in [(2, 1), (-1, 1), (0, -1)]:
        with pytest.raises(rosa.RosaError):
            rosa.kv_bytes(PI0_SHAPE, "bf16", fmt, P)
    lib, cfg = rosa.load(), rosa.model_config(PI0_SHAPE, "bf16")
    cfg.head_dim = 48
    assert lib.rosa_kv_bytes(C.byref(cfg), 0, 1) == -1 and lib.rosa_kv_bytes(None, 0, 1) == -1


def _status(f, *args):
    try:
        f(*args)
    except rosa.RosaError as e:
        assert str(e) and e.status != rosa.ROSA_OK
        return e.status
    return rosa.ROSA_OK


M1 = rosa.ROSA_E_INVALID


@pytest.mark.parametrize("call", [rosa.kv_quantize, rosa.kv_expand])
def test_conversion_refusals(call):
    ok = (A, A + (1 << 20), A + (2 << 20), A + (3 << 20), 16)
    big = 1 << 40
    cases = [
        [(None, *ok[1:])], [(ok[0], None, *ok[2:])], [(*ok[:2], None, *ok[3:])], [(*ok[:3], None, 16)],
        [(ok[0] + 8, *ok[1:])], [(*ok[:3], ok[3] + 2, 16)], [(*ok[:4], -1)],
        [(A, A, A + 16, big, 16)],                                  # destination inside its source
        [(A, A, big, big, 16)],                                     # one destination twice
        [(A, A, big, 2 * big, 16), (A, A, big, 3 * big, 16)],       # shared by two jobs
        [(A, A, big, 2 * big, 16), (big + 16, A, 4 * big, 3 * big, 16)],   # another job's source
    ]
    for jobs in cases:
        assert _status(call, TINY_SHAPE, "bf16", rosa.kv_jobs(jobs), 0) == M1, jobs
    assert _status(call, TINY_SHAPE, "bf16", rosa.kv_jobs([]), 0) == rosa.ROSA_OK
    assert _status(call, TINY_SHAPE, "bf16", rosa.kv_jobs([(None, None, None, None, 0)] * 3), 0) == rosa.ROSA_OK
    arr, _ = rosa.kv_jobs([ok])
    assert _status(call, TINY_SHAPE, "bf16", (arr, -1), 0) == M1
    arr[0].reserved = 1
    assert _status(call, TINY_SHAPE, "bf16", (arr, 1), 0) == M1
    assert _status(call, TINY_SHAPE, "bf16", (None, 1), 0) == M1
    assert _status(call, dataclasses.replace(TINY_SHAPE, head_dim=48), "bf16", rosa.kv_jobs([ok]), 0) == rosa.ROSA_E_UNSUPPORTED


def test_eviction_refusals():
    big = 1 << 40
    base = dict(src_k=A, src_v=A + (1 << 20), dst_k=big, dst_v=2 * big, mass=3 * big, kept=4 * big, kept_mass=5 * big,
                prefix_len=16, keep=8, first=2, last=3)

    def st(fmt=0, **kw):
        return _status(rosa.kv_evict, TINY_SHAPE, "bf16", fmt, rosa.kv_evict_jobs([tuple({**base, **kw}.values())]), 0)
    for kw in [dict(src_k=None), dict(src_v=A + 4), dict(dst_k=None), dict(dst_v=2 * big + 8), dict(mass=None), dict(kept=None),
               dict(kept=4 * big + 2), dict(kept_mass=5 * big + 1), dict(keep=17), dict(keep=4), dict(keep=-1), dict(first=-1),
               dict(last=-1), dict(prefix_len=-1), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
               dict(dst_k=A), dict(dst_v=big), dict(kept=big), dict(kept_mass=3 * big), dict(kept=2 * big + 64)]:
        assert st(**kw) == M1, kw
    assert st(fmt=2) == M1 and st(fmt=-1) == M1
    nothing = dict.fromkeys(["src_k", "src_v", "dst_k", "dst_v", "mass", "kept", "kept_mass"])
    assert st(**nothing, keep=0, first=0, last=0) == rosa.ROSA_OK
    assert st(**nothing, prefix_len=0, keep=0, first=0, last=0) == rosa.ROSA_OK


def test_handle_refusals_before_the_gpu_is_touched():
    lib = rosa.load()
    cfg, cap, h = rosa.model_config(TINY_SHAPE, "bf16"), rosa.capacity(2, 8, 16, 4, 200), C.c_void_p()
    assert lib.rosa_kv_create(None, C.byref(cap), None, C.byref(h)) == M1
    assert lib.rosa_kv_create(C.byref(cfg), None, None, C.byref(h)) == M1
    assert lib.rosa_kv_create(C.byref(cfg), C.byref(cap), None, None) == M1
    assert lib.rosa_kv_create(C.byref(cfg), C.byref(rosa.capacity(0, 8, 16, 4, 200)), None, C.byref(h)) == M1
    assert lib.rosa_kv_create(C.byref(cfg), C.byref(rosa.capacity(2, 2 ** 31 - 1, 16, 4, 200)), None, C.byref(h)) \
        == rosa.ROSA_E_UNSUPPORTED
    assert not h.value and lib.rosa_kv_last_error(None)
    cfg.n_kv_heads = 3
    assert lib.rosa_kv_create(C.byref(cfg), C.byref(cap), None, C.byref(h)) == rosa.ROSA_E_UNSUPPORTED
    assert lib.rosa_kv_plan(None, None, 0, 0, None) == M1
    assert lib.rosa_kv_attention(None, 0, None, None, None) == M1
    assert lib.rosa_kv_mass(None, 0, None, None, 0) == M1
    lib.rosa_kv_destroy(None)
    assert lib.rosa_generate_kv(None, None, 0, 1, 0, None) == M1
