"""The KV cache in 8 bits: sealing, reading back and tree attention behind it, against their definitions in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

from cache_util import DEV, attention_reference, block_values, cache_values, caches, context, tree_parent
from paper_2402_05109_amd import binding as hb

pytestmark = pytest.mark.gpu


def random_kv(seed, B, slots, H, Dh, spread=0.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(B, slots, 2, H, Dh, generator=g, device=DEV)
    return (x * torch.exp(spread * torch.randn(2, H, Dh, generator=g, device=DEV))).half()


def assert_equal(got, want):
    off = (got != want).nonzero()
    assert len(off) == 0, f"{len(off)} values differ, the first at {off[0].tolist()}: {got[tuple(off[0])].item()!r}, not {want[tuple(off[0])].item()!r}"


def fill(c, kv8, kv, L, layer=0, sealed_at=None):
    """Writes the slots to the 16-bit tail and seals what is whole at lengths sealed_at (default L)."""
    B, slots = kv.shape[:2]
    c.kv_write(B, layer, kv8.tail, 0, slots, kv.float().contiguous())
    n = torch.tensor(sealed_at if sealed_at is not None else L, dtype=torch.int32, device=DEV)
    c.hydra_kv8_seal(B, n, kv8)
    return torch.tensor(L, dtype=torch.int32, device=DEV)


def spoil(kv8, NL, H, Dh, sealed, tail_table):
    """NaN into the 16-bit pages of sealed slots: attention must not look at them any more."""
    k = kv8.tail.k_pages.view(NL, -1, H * 16 * Dh)
    v = kv8.tail.v_pages.view(NL, -1, H * 16 * Dh)
    for b, n in enumerate(sealed):
        p = tail_table[b, :n].long()
        k[:, p] = math.nan
        v[:, p] = math.nan


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H,Dh,NL", [(2, 64, 1), (3, 128, 3), (40, 128, 1)])
def test_sealed_values_are_the_definition_bit_for_bit(fmt, H, Dh, NL):
    B, slots = 3, 16 * 5
    L = [79, 33, 15]
    c = context(H, Dh, B, 1, NL)
    kv8 = caches(H, Dh, B, NL, slots, fmt, seed=3)
    kv = [random_kv(10 + l, B, slots, H, Dh) for l in range(NL)]
    # blocks of zeros, of one tiny value, of the largest half, of exact ties (int8: 127 of them make the scale 1)
    kv[0][0, 0:16] = 0.0
    kv[0][0, 16:32] = 0.0
    kv[0][0, 20, :, 0, 5] = 2.0 ** -24
    kv[0][0, 32:48, 0] = 65504.0
    kv[0][0, 48:64] = (torch.arange(16 * Dh, device=DEV).reshape(16, 1, 1, Dh) % 254 / 2.0 - 63.0).half()
    kv[0][0, 63, :, :, Dh - 1] = 127.0
    for l in range(NL):
        c.kv_write(B, l, kv8.tail, 0, slots, kv[l].float().contiguous())
    c.hydra_kv8_seal(B, torch.tensor(L, dtype=torch.int32, device=DEV), kv8)
    assert kv8.n_sealed.tolist() == [n // 16 for n in L] and c.read_flags() == 0
    out = torch.full((NL, B, slots, 2, H, Dh), math.nan, device=DEV)
    c.kv8_read(B, -1, kv8, 0, slots, out)
    for l in range(NL):
        want, _ = cache_values(kv[l], [n // 16 for n in L], fmt)
        assert_equal(out[l].double(), want)
        for b in range(B):
            for i in range(L[b] // 16):
                x = kv[l][b, 16 * i:16 * i + 16].permute(1, 2, 0, 3)
                _, s = block_values(x, fmt)
                assert torch.equal(kv8.scales[l, int(kv8.page_table[b, i])].double(), s.T)
    one = torch.full((B, 21, 2, H, Dh), math.nan, device=DEV)                       # a range that starts and ends inside pages
    c.kv8_read(B, NL - 1, kv8, 7, 21, one)
    assert torch.equal(one, out[NL - 1][:, 7:28])


def check_attention(c, kv8, kv, q, L, sealed, fmt, parent, seed=0):
    B, T = q.shape[:2]
    out = torch.full_like(q, math.nan)
    n = torch.tensor(L, dtype=torch.int32, device=DEV)
    c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, out)
    values, sv = cache_values(kv, sealed, fmt)
    ref, tol = attention_reference(q, values, sv, L, parent)
    assert c.read_flags() == 0
    err = (out.double() - ref).abs()
    assert torch.isfinite(out).all()
    worst = float((err / tol).max())
    assert worst <= 1.0, f"{worst} times what the roundings allow"
    return out


ATTENTION = [
    # H, Dh, T, lengths
    (2, 64, 1, [0, 1, 15]), (2, 64, 1, [16, 17, 31]), (1, 128, 1, [32, 33, 47]), (2, 128, 5, [0, 16, 300]), (4, 64, 31, [48, 63, 64]),
    (2, 128, 32, [31, 32, 700]), (2, 128, 33, [0, 5, 640]), (3, 128, 64, [777, 16, 40]), (2, 64, 64, [1000, 1, 95]), (2, 128, 65, [33, 160, 0]),
    (2, 64, 97, [80, 500, 31]), (2, 128, 128, [0, 144, 1203]), (1, 128, 7, [5003, 4999, 2]), (2, 64, 50, [5000, 17, 2500]),
]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H,Dh,T,L", ATTENTION)
def test_attention_behind_an_8_bit_cache(fmt, H, Dh, T, L):
    B, slots = len(L), max(L) + T
    parent = tree_parent(T)
    c = context(H, Dh, B, T, 1, slots + 8)
    kv8 = caches(H, Dh, B, 1, slots, fmt, seed=T)
    kv = random_kv(T, B, slots, H, Dh)
    fill(c, kv8, kv, L)
    sealed = [n // 16 for n in L]
    spoil(kv8, 1, H, Dh, sealed, kv8.tail.page_table)
    # what lies behind the last node of a row was never written by it
    q = (1.5 * torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(T + 1), device=DEV)).half()
    a = check_attention(c, kv8, kv, q, L, sealed, fmt, parent)
    kv8.tail.seq_len_hint = max(L)
    b = check_attention(c, kv8, kv, q, L, sealed, fmt, parent)
    assert torch.allclose(a.float(), b.float(), rtol=2e-2, atol=2e-2)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("behind", [1, 3, 12])
def test_pages_that_are_not_sealed_yet_are_read_from_the_tail(fmt, behind):
    H, Dh, T, L = 2, 128, 20, [420, 333]
    parent = tree_parent(T)
    c = context(H, Dh, 2, T, 1, 512)
    kv8 = caches(H, Dh, 2, 1, 480, fmt, seed=behind)
    kv = random_kv(behind, 2, 480, H, Dh)
    at = [n - 16 * behind for n in L]
    fill(c, kv8, kv, L, sealed_at=at)
    q = torch.randn(2, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).half()
    check_attention(c, kv8, kv, q, L, [n // 16 for n in at], fmt, parent)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_pages_of_very_different_size(fmt):
    """Scales of K and V that differ by 2^20 from page to page, blocks of zeros, and a row whose weight lies on the page of the smallest values."""
    H, Dh, T, B, L = 2, 128, 33, 2, [350, 217]
    parent = tree_parent(T)
    kv = random_kv(5, B, 400, H, Dh).float()
    for i in range(25):
        kv[:, 16 * i:16 * i + 16, 1] *= 2.0 ** ((i * 7) % 21 - 12)
        kv[:, 16 * i:16 * i + 16, 0] *= 2.0 ** (-((i * 5) % 11))
    kv[:, 64:80] = 0.0
    kv[:, 96:112, 0] = 6.0                                                # a page that the first queries look at alone
    kv[:, 96:112, 1] *= 2.0 ** -6
    kv = kv.half()
    q = torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    q[:, :8] = 3.0
    c = context(H, Dh, B, T, 1, 512)
    kv8 = caches(H, Dh, B, 1, 400, fmt, seed=9)
    fill(c, kv8, kv, L)
    check_attention(c, kv8, kv, q.half(), L, [n // 16 for n in L], fmt, parent)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_sharp_scores(fmt):
    """Scores of some hundreds: one key takes nearly all of the weight."""
    H, Dh, T, B, L = 2, 64, 64, 1, [900]
    parent = tree_parent(T)
    kv = random_kv(6, B, 970, H, Dh)
    q = (60.0 * torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)).half()
    c = context(H, Dh, B, T, 1, 1024)
    kv8 = caches(H, Dh, B, 1, 970, fmt, seed=10)
    fill(c, kv8, kv, L)
    check_attention(c, kv8, kv, q, L, [n // 16 for n in L], fmt, parent)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_more_tiles_to_a_wave_than_a_wave_has_page_ids_at_hand(fmt):
    H, Dh, T, B = 32, 64, 3, 8
    L = [9001] * 7 + [8200]
    parent = tree_parent(T)
    c = context(H, Dh, B, T, 1, 9100)
    kv8 = caches(H, Dh, B, 1, 9010, fmt, seed=11)
    kv = random_kv(7, B, 9010, H, Dh)
    fill(c, kv8, kv, L)
    q = torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(4), device=DEV).half()
    check_attention(c, kv8, kv, q, L, [n // 16 for n in L], fmt, parent)


def test_rows_out_of_range_are_flagged_and_left_alone():
    H, Dh, T, B = 2, 64, 4, 4
    L = [100, 100, 100, 100]
    parent = tree_parent(T)
    c = context(H, Dh, B, T, 1, 128)
    kv8 = caches(H, Dh, B, 1, 112, "int8", seed=12)
    kv = random_kv(8, B, 112, H, Dh)
    n = fill(c, kv8, kv, L)
    q = torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).half()
    good = check_attention(c, kv8, kv, q, L, [6] * B, "int8", parent)
    kv8.n_sealed.copy_(torch.tensor([6, 7, -1, 6], dtype=torch.int32))    # more than are whole; negative
    n[3] = 111                                                            # the nodes do not fit the table
    out = torch.full_like(q, 7.0)
    c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, out)
    assert torch.equal(out[0], good[0]) and bool((out[1:] == 7.0).all())
    assert c.read_flags() == 1
    # a page of the codes outside the pool: flagged, no access outside
    kv8.n_sealed.copy_(torch.tensor([6, 6, 6, 6], dtype=torch.int32))
    kv8.page_table[1, 2] = 10 ** 6
    n[3] = 100
    c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, out)
    assert torch.equal(out[0], good[0]) and torch.equal(out[2:], good[2:]) and c.read_flags() == 64
    # sealing: the row with the bad entry keeps its n_sealed, so does one whose n_sealed is out of range
    kv8.n_sealed.copy_(torch.tensor([0, 0, 9, 6], dtype=torch.int32))
    c.hydra_kv8_seal(B, n, kv8)
    assert kv8.n_sealed.tolist() == [6, 0, 9, 6] and c.read_flags() == 1 | 64


def test_other_streams_and_graphs():
    H, Dh, T, B, L = 2, 128, 40, 2, [300, 213]
    parent = tree_parent(T)
    c = context(H, Dh, B, T, 1, 512)
    kv8 = caches(H, Dh, B, 1, 352, "int8", seed=13)
    kv = random_kv(9, B, 352, H, Dh)
    n = fill(c, kv8, kv, L)
    q = torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(6), device=DEV).half()
    want = check_attention(c, kv8, kv, q, L, [x // 16 for x in L], "int8", parent)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, out)
    side.synchronize()
    assert torch.equal(out, want)
    start = torch.zeros_like(kv8.n_sealed)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv8.n_sealed.copy_(start)
        c.hydra_kv8_seal(B, n, kv8)
        c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, out)
    for i in range(4):
        out.zero_()
        kv8.scales.zero_()
        q2 = torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(20 + i), device=DEV).half()
        q.copy_(q2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kv8.n_sealed, n // 16)
        got = out.clone()
        check = check_attention(c, kv8, kv, q, L, [x // 16 for x in L], "int8", parent)
        assert torch.equal(got, check)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H,Dh,B", [(2, 128, 1), (32, 64, 9)])             # few rows; more (row, head)s than compute units
@pytest.mark.parametrize("small,large", [(160, 416), (416, 160)])
@pytest.mark.parametrize("down", [10, 16, 20])
def test_weight_shared_by_pages_of_large_and_small_values(fmt, H, Dh, B, small, large, down):
    """Two pages of one wave's tiles take equal shares of the weight, and the values of one are 2^-down of the other's: the small ones do not show in
    the result, but their weight does, in the sum that it is divided by."""
    T, L = 8, [700] * B
    parent = tree_parent(T)
    kv = random_kv(21, B, 720, H, Dh).float()
    kv[:, :, 0] *= 0.05
    direction = torch.randn(H, Dh, generator=torch.Generator(device=DEV).manual_seed(7), device=DEV)
    kv[:, small:small + 16, 0] = direction
    kv[:, large:large + 16, 0] = direction
    kv[:, :, 1] *= 100.0
    kv[:, small:small + 16, 1] *= 2.0 ** -down
    kv = kv.half()
    q = direction.expand(B, T, H, Dh).half().contiguous()
    c = context(H, Dh, B, T, 1, 1024)
    kv8 = caches(H, Dh, B, 1, 720, fmt, seed=22)
    fill(c, kv8, kv, L)
    check_attention(c, kv8, kv, q, L, [n // 16 for n in L], fmt, parent)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("T", [1, 33, 128])
def test_nothing_sealed(fmt, T):
    H, Dh, L = 2, 64, [1500, 3]
    parent = tree_parent(T)
    c = context(H, Dh, 2, T, 1, 1700)
    kv8 = caches(H, Dh, 2, 1, 1500 + T, fmt, seed=T)
    kv = random_kv(T, 2, 1500 + T, H, Dh)
    fill(c, kv8, kv, L, sealed_at=[0, 0])
    q = torch.randn(2, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).half()
    check_attention(c, kv8, kv, q, L, [0, 0], fmt, parent)
    kv8.tail.seq_len_hint = 1500
    check_attention(c, kv8, kv, q, L, [0, 0], fmt, parent)
    kv8.tail.seq_len_hint = 1                                # a hint that is too short: never a matter of results
    check_attention(c, kv8, kv, q, L, [0, 0], fmt, parent)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_caches_beyond_4_gib(fmt):
    """Pages whose codes, and whose 16-bit values, lie more than 2^32 bytes behind the first ones."""
    H, Dh, T, B, L = 8, 128, 9, 2, [150, 97]
    more = 2 ** 32 // (H * 16 * Dh) + 5
    parent = tree_parent(T)
    c = context(H, Dh, B, T, 1, 256)
    kv8 = caches(H, Dh, B, 1, 176, fmt, seed=30, more=more)
    kv = random_kv(30, B, 176, H, Dh)
    fill(c, kv8, kv, L)
    spoil(kv8, 1, H, Dh, [n // 16 for n in L], kv8.tail.page_table)
    q = torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).half()
    check_attention(c, kv8, kv, q, L, [n // 16 for n in L], fmt, parent)
    # the sealed pages of row 0 moved to the front
    was = kv8.page_table[0, :9].clone()
    to = torch.arange(9, dtype=torch.int32, device=DEV)
    c.hydra_kv8_copy_pages(kv8, 9, was, to)
    kv8.page_table[0, :9] = to
    check_attention(c, kv8, kv, q, L, [n // 16 for n in L], fmt, parent)
    out = torch.full((B, 64, 2, H, Dh), math.nan, device=DEV)
    c.kv8_read(B, 0, kv8, 20, 64, out)
    want, _ = cache_values(kv, [n // 16 for n in L], fmt)
    assert_equal(out.double(), want[:, 20:84])
    tail = kv8.tail.page_table[1, 6:7].clone()
    c.hydra_kv_copy_pages(kv8.tail, 1, tail, to[:1])
    block = H * 16 * Dh
    assert torch.equal(kv8.tail.k_pages[:block], kv8.tail.k_pages[int(tail) * block:(int(tail) + 1) * block]) and c.read_flags() == 0


@pytest.mark.parametrize("H,B", [(2, 1), (32, 9)])                          # all keys in one workgroup; keys split over waves
@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 3, -2 ** 31])
def test_lengths_at_the_ends_of_the_integers(H, B, length):
    """Such a row is left alone and flagged; the others are what they would be without it."""
    Dh, T = 64, 4
    c = context(H, Dh, B, T, 1, 128)
    kv8 = caches(H, Dh, B, 1, 112, "int8", seed=2)
    n = fill(c, kv8, random_kv(3, B, 112, H, Dh), [100] * B)
    q = torch.randn(B, T, H, Dh, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).half()
    want = torch.zeros_like(q)
    c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, want)
    n[B - 1] = length
    out = torch.full_like(q, 7.0)
    c.tree_attention_kv8(B, 0, c.ws, q, n, kv8, out)
    assert torch.equal(out[:B - 1], want[:B - 1]) and bool((out[B - 1] == 7.0).all())
    c.hydra_kv8_seal(B, n, kv8)
    assert kv8.n_sealed.tolist() == [6] * B and c.read_flags() == 1
