"""The sizes that attention over a paged cache takes, as its header states them (host checks alone: no
call here reaches the device, for its workspace is too small)."""
import itertools

import pytest

from test_cache_cpu import BAD_DIM, WORKSPACE, attend
from paper_2002_00876_amd import binding


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def _tiles(N, Hq, Hk):
    return -(-N * Hq // (64 * Hk))


@pytest.mark.parametrize("B", [1, 3, 32, 255, 256])
@pytest.mark.parametrize("N,Hq,Hk", [(1, 1, 1), (256, 1, 1), (1, 512, 512), (1, 600, 600), (1, 1024, 1024), (7, 1024, 64),
                                     (256, 1024, 4), (65, 8, 8)])
def test_up_to_the_stated_number_of_slots_fits(L, B, N, Hq, Hk):
    # B ceil(N Hq / (64 Hk)) M S up to 2^35, whatever M and S
    if B * N * Hq > 1 << 29:
        pytest.skip("more rows than a call takes")
    most = min((1 << 35) // (B * _tiles(N, Hq, Hk)), 1 << 30)
    for S, odd in itertools.product((1, 7, 16, 1 << 15, most), (0, 1)):
        M = most // S - odd
        if M >= 1:
            got = attend(L, B=B, N=N, Hq=Hq, Hk=Hk, S=S, M=M, nb=0)
            assert got == WORKSPACE, (S, M, L.ts_last_error().decode())


def test_far_beyond_it_is_refused(L):
    assert attend(L, B=256, Hk=600, Hq=600, N=1, S=1 << 15, M=1 << 15) == BAD_DIM
    assert attend(L, B=256, Hk=1024, Hq=1024, N=256, S=1 << 20, M=1 << 10) == BAD_DIM
