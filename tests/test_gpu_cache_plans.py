"""Masses over 4-bit caches where one block of sixteen waves takes a whole sequence: heads for which its scores are beside it in
LDS and for which they are not, many blocks and few, windows of as many tokens."""
import pytest

from tests.test_gpu_cache_attend import _check_mass, _data

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("lengths,hq,hk,d,page,t,window", [
    ([768 - 3 * i for i in range(32)], 32, 2, 128, 16, BF, 0), ([705, 1, 0], 36, 4, 128, 32, BF, 0),
    ([705 - i for i in range(16)], 36, 4, 128, 50, F16, 0), ([544, 513, 300], 16, 1, 128, 16, F16, 0),
    ([545 - i for i in range(64)], 13, 1, 128, 64, BF, 0), ([768], 48, 3, 96, 32, BF, 0), ([768, 767], 16, 1, 64, 16, F16, 0),
    ([3000, 760, 20], 64, 4, 128, 16, BF, 700), ([2000 - 7 * i for i in range(20)], 64, 4, 128, 64, BF, 600), ([640, 639], 10, 1, 128, 7, BF, 0)])
def test_one_block_of_sixteen_waves(lengths, hq, hk, d, page, t, window):
    print(f"mass {len(lengths)} sequences of up to {max(lengths)}, heads={hq}/{hk} d={d} page={page} {t} window={window}", flush=True)
    a = _data(lengths, hq, hk, d, page, t)
    _check_mass(a, window=window)
    _check_mass(a, window=window, span=max(lengths) + 5)
