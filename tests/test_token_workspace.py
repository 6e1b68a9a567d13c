"""CPU-only: a workspace sized for the largest call serves every smaller one."""
import pytest

from paper_2002_06015_amd import kfac

COUNTS = sorted({max(0, c + d) for c in (0, 1, 8, 64, 2048, 8192, 16384, 32768, 65536, 100000, 131072, 524288, 1 << 20, 1 << 24) for d in (-1, 0, 1, 7)})
KEYS = sorted({c + d for c in (2, 3, 32, 64, 256, 512, 1024, 32000, 1 << 17, 1 << 18, 1 << 19, 1 << 24, 1 << 27, (1 << 30) - 2) for d in (-1, 0, 1)})


def _never_falls(sizes, what):
    for (a, u), (b, v) in zip(sizes, sizes[1:]):
        assert 0 < u <= v, "%s: %s needs %d bytes, %s needs %d" % (what, a, u, b, v)


@pytest.mark.parametrize("num", [1, 16, 511, 512, 32000, 1 << 20])
def test_more_positions_need_no_less(num):
    _never_falls([(n, kfac.kfac_segments_workspace_bytes(n, num)) for n in COUNTS], "segments of %d keys" % num)
    for dim in (1, 100, 1024):
        _never_falls([(n, kfac.kfac_embedding_workspace_bytes(n, num, dim)) for n in COUNTS], "embedding of %d x %d" % (num, dim))


@pytest.mark.parametrize("n", [0, 5, 8192, 8193, 50000, 1 << 20])
def test_more_keys_need_no_less(n):
    _never_falls([(k, kfac.kfac_segments_workspace_bytes(n, k)) for k in KEYS], "segments of %d positions" % n)
    for dim in (1, 100):
        _never_falls([(k, kfac.kfac_embedding_workspace_bytes(n, k, dim)) for k in KEYS], "embedding of %d positions" % n)


def test_longer_rows_need_no_less():
    for n in (100, 32768, 32769):
        _never_falls([(d, kfac.kfac_embedding_workspace_bytes(n, 5000, d)) for d in range(1, 300)], "embedding of %d positions" % n)
