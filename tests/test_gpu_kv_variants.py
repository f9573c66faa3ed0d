"""GPU tests of the prefix-cache kernels where their variants meet: items of few
query rows (their waves take different keys) and of more, blocks of few and of
many keys in the masses, evicted rows longer than the part held on chip, and
masses that two requests would share."""
import dataclasses

import numpy as np
import pytest

from oracle import kv as okv
from synthetic import PI0_SHAPE
from tests.test_gpu_kv import (ALT64_SHAPE, ALT256_SHAPE, HD64_SHAPE, HD256_SHAPE, SHAPES, Batch, Guarded, check_batch, check_mass,
                               evict_case, gen, run_batch)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# 7 query heads to the KV head: no stage of 32 or 64 rows is whole tokens
G7_SHAPE = dataclasses.replace(PI0_SHAPE, n_layers=2, n_q_heads=14, n_kv_heads=2, head_dim=64)

EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 96, 97, 127, 128, 129, 160, 257, 300]


@pytest.mark.parametrize("fmt", [0, 1], ids=["model", "fp4"])
@pytest.mark.parametrize("shape", [*SHAPES, "g7"])
def test_few_query_rows_at_every_edge_of_their_key_tiles(shape, fmt):
    s = G7_SHAPE if shape == "g7" else SHAPES[shape]
    G = s.n_q_heads // s.n_kv_heads
    few = max(1, 16 // G)
    # most rows an item of few rows has, one, and one token more than it may have
    specs = [(P, (1, few, few + 1)[i % 3]) for i, P in enumerate(EDGES)] + [(3000, 1), (3001, few)]
    for layer in range(2):
        b = Batch(s, "bf16", fmt, specs, seed=21 + layer)
        run_batch(b, layer).close()
        o, lse = b.out()
        check_batch(b, layer, o, lse)
        assert b.o.intact() and b.lse.intact()
        if not (s.attention_layout == 1 and layer % 2):
            check_mass(b, layer)


@pytest.mark.parametrize("layout", [HD64_SHAPE, HD256_SHAPE, ALT64_SHAPE, ALT256_SHAPE],
                         ids=["joint64", "joint256", "alternating64", "alternating256"])
def test_one_token_without_a_prefix_or_with_its_own_keys_only(layout):
    joint = layout.attention_layout == 0
    specs = [(0, 1), (0, 2), (40, 1)] if joint else [(40, 1), (33, 2), (7, 1)]
    for layer in range(2):
        b = Batch(layout, "bf16", 1, specs, seed=3)
        run_batch(b, layer).close()
        check_batch(b, layer, *b.out())


@pytest.mark.parametrize("fmt", [0, 1], ids=["model", "fp4"])
def test_few_rows_with_scores_that_rise(fmt):
    def shift(i, x):
        ramp = torch.linspace(0.1, 30.0, x.shape[1], device="cuda")
        return (x.float() * (ramp if i % 2 == 0 else ramp.flip(0))[None, :, None, None]).to(x.dtype)
    for shape in (HD256_SHAPE, HD64_SHAPE, G7_SHAPE):
        b = Batch(shape, "bf16", fmt, [(700, 1), (90, 2), (400, 1), (2100, 1), (33, 1)], seed=9, shift=shift)
        run_batch(b, 0).close()
        check_batch(b, 0, *b.out())
        check_mass(b, 0)


@pytest.mark.parametrize("fmt", [0, 1], ids=["model", "fp4"])
@pytest.mark.parametrize("shape", ["hd32", "hd64", "hd128", "hd256", "g7"])
def test_masses_of_many_requests_in_blocks_of_many_keys(shape, fmt):
    s = G7_SHAPE if shape == "g7" else SHAPES[shape]
    special = [(1, 1), (256, 9), (257, 33), (511, 50), (700, 3), (31, 70), (512, 17)]
    # at least 256 blocks of 256 keys and KV head
    specs = special + [(1 + 37 * i % 300, 1 + i % 3) for i in range(260)]
    b = Batch(s, "bf16", fmt, specs, seed=31)
    h = run_batch(b, 1)
    which = [*range(len(special)), 100, len(specs) - 1]
    check_mass(b, 1, which=which)
    h.mass(1, b.qkv, b.lse.all)                    # again, added
    torch.cuda.synchronize()
    check_mass(b, 1, times=2, which=which)
    for m in b.mass:
        assert bool((m[0] == 7.0).all()) and bool(torch.isfinite(m[1]).all())
    h.close()


def test_masses_have_the_same_bits_every_time():
    for specs in ([(816, 50), (33, 1)], [(20 + i, 16) for i in range(300)]):
        b = Batch(HD64_SHAPE, "bf16", 1, specs, seed=4)
        run_batch(b, 0).close()
        first = [m.clone() for m in b.mass]
        run_batch(b, 0).close()
        assert all(torch.equal(x, y) for x, y in zip(first, b.mass))


def test_masses_of_two_requests_may_not_share_memory():
    from paper_2607_01088_amd import rosa
    b = Batch(HD64_SHAPE, "bf16", 1, [(64, 1), (64, 2)], seed=5)
    h = rosa.KvAttention(b.shape, b.dtype, b.cap)
    good = b.mass
    n = good[0].numel()
    both = torch.empty(2 * n, device="cuda")

    def refused(mass):
        with pytest.raises(rosa.RosaError) as e:
            h.plan(b.structs, 1, mass=mass)
        return e.value.status == rosa.ROSA_E_INVALID
    assert refused([good[0], good[0]])                                   # the same array twice
    assert refused([both[:n], both[n - 1:]])                             # one element in common
    assert refused([b.keep[1][0], good[1]])                              # a cache in the place of masses
    h.plan(b.structs, 1, mass=[both[:n], both[n:]])                      # side by side
    twice = [b.structs[0], b.structs[0]]                                 # one cache for two requests
    h.plan(twice, 1, mass=good)
    h.close()


def test_outputs_that_overlap_are_refused():
    from paper_2607_01088_amd import rosa
    b = Batch(HD64_SHAPE, "bf16", 1, [(64, 3), (10, 2)], seed=5)
    h = rosa.KvAttention(b.shape, b.dtype, b.cap)
    h.plan(b.structs, 1)
    qkv, o, lse = b.qkv, b.o.all, b.lse.all
    n = b.qkv.numel() * 2
    room = torch.empty(2 * n + 4096, dtype=torch.uint8, device="cuda")
    room[:n] = qkv.view(torch.uint8).flatten()
    for bad in ((qkv, qkv, lse), (qkv, o, qkv), (qkv, o, o), (room[:n], room[n - 16:], lse)):
        with pytest.raises(rosa.RosaError) as e:
            h.attention(0, bad[0], bad[1], lse=bad[2])
        assert e.value.status == rosa.ROSA_E_INVALID
    h.attention(0, room[:n], room[n:], lse=lse)                          # side by side
    h.attention(0, qkv, o, lse=None)
    torch.cuda.synchronize()
    check_batch(b, 0, b.out()[0], None)
    assert torch.equal(room[n:n + b.o.n], b.o.data)
    h.close()


@pytest.mark.parametrize("fmt", [0, 1], ids=["model", "fp4"])
def test_eviction_from_long_rows(fmt):
    specs = [(12287, 5000, 4, 48), (12288, 1, 0, 0), (12289, 12288, 0, 0), (20001, 15000, 4, 48), (40000, 100, 0, 3), (4096, 17, 1, 1),
             (4097, 4000, 0, 0)]

    def masses(i, m):
        return (m * 8).round() if i % 2 else m                           # ties across the whole row
    evict_case(SHAPES["hd32"], "bf16", fmt, specs, seed=12, masses=masses)
    evict_case(SHAPES["hd32"], "bf16", fmt, specs[-2:], seed=13, masses=masses)
