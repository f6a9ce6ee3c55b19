"""What the workspace queries of the cache's attention say is enough for the calls, of every kind of cache.

No launch happens: these run where no GPU is, and a call that passes all checks ends with CP_ERR_HIP."""
import ctypes
import itertools
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls with made-up addresses must not reach a GPU")

BF16, E4M3, E2M1 = 1, 3, 4
WORKSPACE, HIP = 3, 4
FAKE = ctypes.c_void_p(1 << 36)
HEADS = [1, 2, 3, 4, 7, 8, 9, 10, 11, 12, 13, 14, 15, 16, 17, 20]
LENGTHS = [1, 32, 480, 512, 513, 540, 544, 545, 600, 640, 673, 705, 736, 737, 760, 768, 769, 800, 1000, 1024, 1025, 1500, 5000, 131072]


@pytest.fixture(scope="module")
def lib():
    import paper_2608_13226_amd as cp
    if not os.path.exists(cp.library_path()):
        from paper_2608_13226_amd import build
        build.build()
    return cp.library()


def _cases(d):
    for group, (batch, hk), (longest, window) in itertools.product(
            HEADS, [(1, 1), (1, 4), (15, 4), (16, 4), (49, 4), (63, 1), (64, 1), (32, 2), (200, 8)],
            [(n, 0) for n in LENGTHS] + [(5000, w) for w in (480, 500, 544, 600, 700, 736, 737, 768)]):
        yield batch, group * hk, hk, d, longest, window


@pytest.mark.parametrize("held", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_masses(lib, d, held):
    scale = FAKE if held == E2M1 else None
    for batch, hq, hk, d, longest, window in _cases(d):
        size = lib.coverprune_paged_attention_mass_workspace(batch, hq, hk, d, longest, window)
        code = lib.coverprune_paged_attention_mass(FAKE, BF16, batch, hq, hk, d, FAKE, FAKE, held, 100, 16, scale, scale, FAKE, 10000, FAKE,
                                                   longest, window, 0.1, FAKE, longest, FAKE, None, FAKE, size, None)
        assert code == HIP, (batch, hq, hk, d, longest, window, size, lib.coverprune_last_error())


@pytest.mark.parametrize("held", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_attention(lib, d, held):
    for batch, hq, hk, d, longest, window in _cases(d):
        size = lib.coverprune_paged_attention_workspace(batch, hq, hk, d, longest, window)
        rest = (FAKE, 10000, FAKE, longest, window, 0.1, FAKE, None, FAKE, size, None)
        if held == E2M1:
            code = lib.coverprune_paged_attention4(FAKE, BF16, batch, hq, hk, d, FAKE, FAKE, 100, 16, FAKE, FAKE, *rest)
        else:
            code = lib.coverprune_paged_attention(FAKE, BF16, batch, hq, hk, d, FAKE, FAKE, held, 100, 16, None, None, *rest)
        assert code == HIP, (batch, hq, hk, d, longest, window, size, lib.coverprune_last_error())


def test_eviction(lib):
    """As much as the query says for any recent; a sink takes none."""
    for (batch, hk), longest, keep in itertools.product([(1, 1), (3, 4), (64, 8)], [1, 1000, 2049, 16384, 16385, 100000], [1, 7, 900, 8000, 50000]):
        for recent in {0, keep // 3, keep}:
            size = lib.coverprune_kv_evict_workspace(batch, hk, keep, recent, longest)
            for sink in {0, keep - recent}:
                code = lib.coverprune_kv_evict(FAKE, FAKE, BF16, 100, 16, hk, 64, None, None, FAKE, batch, 10000, FAKE, longest,
                                               ctypes.c_void_p(2 << 36), longest, keep, recent, sink, FAKE, ctypes.c_void_p(2 << 36),
                                               ctypes.c_void_p(3 << 36), FAKE, size, None)
                assert code == HIP, (batch, hk, longest, keep, recent, sink, size, lib.coverprune_last_error())
