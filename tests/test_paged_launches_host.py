"""How the decode calls over a paged cache in 8 bits spread their rows over the blocks (no GPU; see launches.py)."""
import pytest

import launches
import test_gpu_quant_spread

N_CU = 256  # of the recorder


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("recorder")
    return lambda *steps: launches.run([["create", {}]] + [list(s) for s in steps], tmp)[1:]


def _tiles(n):
    return max(-(-n // 32), 1)


def _rounds(n, launch, hkv=8):
    """(rounds of a block's waves that the longest block takes, rounds that an even share of the blocks at work together takes)."""
    waves = launch["threads"] // 64
    slots = N_CU * (8 // waves)
    return -(-launch["tiles"] // waves), sum(_tiles(x) for x in n) * hkv / slots / waves


UNEVEN = [[400] * a + [long] + [400] * b for a, b, long in ((10, 9, 16000), (14, 13, 16000), (15, 15, 16000), (0, 31, 16000), (31, 0, 16000), (31, 31, 16000),
                                                          (32, 31, 16000), (30, 1, 60000), (15, 16, 2000))] + [
    [500] * 63 + [60000], [500] * 31 + [32768], [100] * 31 + [4000], [100] * 28 + [8000] * 4, [200] * 62 + [3000] * 2, [600] * 15 + [8000] + [600] * 15,
    [0] * 20 + [40000] + [300] * 43]


@pytest.mark.parametrize("n", UNEVEN, ids=lambda n: "%dx%d" % (len(n), max(n)))
def test_a_long_sequence_among_short_ones_is_shared(calls, n):
    """A row's piece takes what an even share of the call takes, half as much again at most (pieces are rounded to whole numbers of a row), and
    two rounds for the short rows' sake (a row of up to 16 tiles stays whole).  In one round of blocks the long row went to one block."""
    got = calls(("decode", {"n": n}))[0]
    assert got["value"] == 0 and launches.kernels(got)[0].startswith("k_decode_quant<")
    longest, even = _rounds(n, got["launches"][0])
    assert longest <= 1.5 * even + 4, (longest, even, got["launches"])


@pytest.mark.parametrize("n,tiles,blocks", [([768] * 20, 24, 160), ([60000] * 7, 469, 224), ([4000] * 12, 63, 192), ([1000] * 24, 32, 192), ([32768], 32, 256),
                                            ([400] * 15 + [1000] + [400] * 16, 32, 256)])
def test_rows_alike_take_one_round(calls, n, tiles, blocks):
    launch = calls(("decode", {"n": n}))[0]["launches"][0]
    assert (launch["tiles"], launch["blocks"]) == (tiles, blocks)


def test_pieces_fit_the_workspace(calls):
    """Two partial results a block: room for 1024 blocks.  And no row has more than 64 pieces."""
    steps = [[short] * (n - 1) + [long] for n in (2, 9, 31, 32, 33, 40, 63, 64) for short in (0, 1, 513, 700, 1100) for long in (600, 5000, 60000, 300000)]
    for n, r in zip(steps, calls(*[("decode", {"n": n}) for n in steps])):
        assert r["value"] == 0 and r["launches"][0]["blocks"] <= 1024, n
        assert 64 * r["launches"][0]["tiles"] >= _tiles(max(n)), n


@pytest.mark.parametrize("case", test_gpu_quant_spread.UNEVEN + test_gpu_quant_spread.REFILL + test_gpu_quant_spread.SHARES, ids=lambda c: "%dx%d" % (len(c[0]), max(c[0])))
def test_cases_take_their_kernel(calls, case):
    ns, hq, hkv, page, _, kernel, tiles = case
    launch = calls(("decode", {"n": ns, "hq": hq, "hkv": hkv, "page": page}))[0]["launches"][0]
    assert launch["kernel"].endswith("k_decode_quant" + kernel) and launch["tiles"] == tiles, launch
