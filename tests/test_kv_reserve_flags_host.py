"""Flags of seer_kv_reserve, without a GPU: unknown ones are refused before anything is launched."""
import ctypes


def test_unknown_flags_are_refused():
    from paper_2511_14617_amd import binding as b
    lib = b.load_library()
    for flags, size in ((0, True), (b.SEER_RESERVE_OWN_PAGES, True), (2, False), (3, False), (-1, False), (-2 ** 31, False)):
        p = b.SeerReserveParams(B=4, page_size=16, num_pages=100, max_pages_per_seq=32, n_tokens=50, flags=flags)
        assert (b.seer_kv_reserve_workspace(p) > 0) == size
        if not size:
            assert lib.seer_kv_reserve(ctypes.byref(p), *[0x1000] * 13, 1 << 40, None) == b.SEER_EINVAL
