"""Which kernels the paged cache and masked attention launch, and with what.  CPU only: the launches are written down, not made."""
import os
import struct

import pytest

import launch_util
from launch_util import P
from paper_2604_12798_amd import build

NULL = 0


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if not os.path.exists(build.LIB) or not os.path.exists(build.BINDING):
        build.build_lib()
    log = launch_util.build(tmp_path_factory.mktemp("launches"))
    return lambda calls: launch_util.launches(log, calls)


ONE, FIXED, DEALT = 0, 1, 2  # what the lengths of a decode's sequences are to its kernel (its third template argument)


def decode(B, Hq, Hkv, page, M, n_splits, n_q=1, d=64, lens=P, n_keys=0):
    return ("vfa_kvp_decode_fwd", [P, P, P, P, P, P, B, Hq, Hkv, 9, page, M, n_q, d, lens, n_keys, n_splits, 0.0, 0.0, NULL, P, 1 << 40, NULL], 0)


def test_ranges_are_dealt_only_where_an_int_counts_the_tiles(launches):
    """Sequences may share pages or miss them, so 128 of 2^30 tokens are a call like others: 2^31 tiles, which an int does not hold.  The search of a range's sequence would
    end at once, all ranges would be those of the first one, and the merge would read entries of the others that nobody wrote."""
    page, M = 1 << 14, 1 << 16
    calls = [decode(B, 1, 1, page, M, 2) for B in (2, 64, 127, 128, 200)] + [decode(64, 1, 1, page, M, 4096), decode(100, 1, 1, page, M // 2, 2)]
    for (rc, made), form in zip(launches(calls), (DEALT, DEALT, DEALT, FIXED, FIXED, DEALT, DEALT)):
        assert rc == 0 and [m[0] for m in made] == ["kvp_decode_kernel", "decode_merge_kernel"]
        assert made[0][1][2] == form and made[1][1][1] == (2 if form == DEALT else 0)


def test_prefixes_are_read_for_causal_documents_only(launches):
    """The header says that prefix_lens is not read for causal = 0, so it may be anything there."""
    made = launches([("vfa_row_ranges", [P, 2 * P, 3 * P, 1, 1000, 2, causal, NULL], 24) for causal in (1, 0)])
    for (rc, [kernel]), prefix in zip(made, (2 * P, 0)):
        assert rc == 0 and kernel[0] == "row_ranges_kernel" and kernel[2] == (4, 1, 1)
        assert struct.unpack("<3Q", kernel[4]) == (P, prefix, 3 * P)


def test_suggested_ranges_are_of_the_form_that_they_are_counted_for(launches):
    """Ranges of lengths on the GPU are counted for workgroups of one wave where they are dealt out, and so they are; else for workgroups of four waves."""
    import paper_2604_12798_amd as vfa
    calls, said = [], []
    for d in (64, 128):
        for Hkv in (1, 2, 8):
            for B in (2, 17, 50, 63, 64, 65, 80, 100, 129, 200, 256, 257, 300):
                for n in (400, 520, 1000, 1500, 2048, 2049, 4096, 4097, 32768):
                    s = vfa.kvp_decode_splits(B, 4 * Hkv, Hkv, 1, d, n, True)
                    said.append((d, Hkv, B, n, s))
                    calls.append(decode(B, 4 * Hkv, Hkv, 16, -(-n // 16), s, d=d))
    for (d, Hkv, B, n, s), (rc, made) in zip(said, launches(calls)):
        assert rc == 0, (d, Hkv, B, n, s)
        four_waves = max(1, 256 * (2 if d == 64 else 1) // (B * Hkv))
        form = made[0][1][2]
        if B <= 256:
            assert (form == DEALT) == (s > 1), (d, Hkv, B, n, s)
        elif n <= 2048:
            assert form == FIXED and s <= four_waves, (d, Hkv, B, n, s)


def test_a_long_sequence_among_many_gets_ranges():
    """Many sequences keep the units busy with one range each, if none of them can be long; else the longest one would have a unit for each of its heads and no more."""
    import paper_2604_12798_amd as vfa
    s = lambda B, n, d=128, Hkv=8: vfa.kvp_decode_splits(B, 4 * Hkv, Hkv, 1, d, n, True)
    for d in (64, 128):
        assert s(64, 4096, d) == 1 and s(128, 1024, d) == 1
        for n in (4097, 8192, 32768):
            assert 2 <= s(64, n, d) <= 4 and s(128, n, d) == 2
        assert s(256, 32768, d) == 1  # (2048 heads: not dealt with more)
        assert 2 <= s(300, 32768, d, 1) and s(300, 1000, d, 1) == 1
    assert s(100, 1000, 128, 1) == 7 and s(80, 1500, 128, 1) == 11
    assert s(16, 8192) == 8 and s(4, 32768) == 32   # (as before)


def prompt(B, Hq, Hkv, N, d, cap=0.0, slopes=NULL):
    return ("vfa_masked_attn_fwd", [P, P, P, P, P, B, Hq, Hkv, N, d, 1, P, 0.0, cap, slopes, NULL], 0)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_a_workgroup_of_masked_attention(launches, d):
    """128 where the units (256 without a GPU) hold no more workgroups of them than there are, two of them each, three at d = 64; else 64.  All kinds of scores."""
    places = 512 if d == 128 else 768
    calls, want = [], []
    for items, blocks in ((places, 1), (places - 1, 1), (places, 4), (places - 4, 4), (5 * places, 5), (1, 1)):
        for cap, slopes in ((0.0, NULL), (30.0, NULL), (0.0, P), (50.0, P)):
            for N in (128 * blocks, 128 * blocks - 127):
                calls.append(prompt(1, items // blocks, 1, N, d, cap, slopes))
                many = items >= places
                want.append(((d, 4, 1) if many else (d, 2, 2)) + (int(cap > 0), int(slopes != NULL)) + (items // blocks * -(-N // (128 if many else 64)),))
    for (rc, made), w in zip(launches(calls), want):
        [(name, form, grid, block, _)] = made
        assert rc == 0 and name == "attn_masked_kernel" and form == w[:5] and grid == (w[5], 1, 1) and block == (256, 1, 1)
