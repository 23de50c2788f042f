"""seer_kv_append where a workgroup takes two or four tokens: small heads, from 2048 and from 4096 tokens on.  Against the rotation in 64 bits with the
tolerance of the other tests of this call."""
import pytest

from test_gpu_kv_append import make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [2047, 2048, 2049, 4095, 4096, 4097, 4098, 4099])
@pytest.mark.parametrize("heads", [(8, 1, 128, 128, 16, 128, 0), (4, 2, 64, 64, 20, 32, 16), (0, 2, 64, 0, 16, 64, 0), (2, 1, 192, 128, 32, 64, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_groups_of_tokens(N, heads, interleaved):
    """Tokens without a slot among the others (a fifth of all, so that most groups of four hold one), the last group cut by every remainder, to q_out and in place."""
    Hq, Hkv, D, Dv, page, R, at = heads
    place = "itself" if N % 2 else "new"
    run(make(N, N, Hq, Hkv, D, Dv, page, N // page + 3, R, at, interleaved, empty=0.2), page, place)


@pytest.mark.parametrize("N", [2051, 4101])
def test_slices_of_one_projection(N):
    run(make(N, N, 8, 1, 128, 128, 16, N // 16 + 3, 64, 32, False, empty=0.3, fused=True), 16)


@pytest.mark.parametrize("N", [2049, 4099])
def test_no_rotation_and_none_live(N):
    run(make(N, N, 2, 2, 64, 64, 16, N // 16 + 3, 0, 0, False, empty=0.5), 16)
    c = make(N, N, 2, 2, 64, 64, 16, N // 16 + 3, 64, 0, False)
    c["slot"].fill_(-1)
    run(c, 16)
