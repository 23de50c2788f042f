"""Host-side checks, without a GPU, of the calls in front of the first verification step: parameter structs, workspace sizes, and bad
arguments turned into SEER_E* codes or refused by the binding before anything is launched."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000       # never dereferenced: all of these calls fail on the host


@pytest.fixture(scope="module")
def lib():
    from paper_2511_14617_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_library()
    return binding.load_library()


def struct_fields(name):
    header = open(os.path.join(ROOT, "include", "seer_verify.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), header, flags=re.S).group(1)
    fields = []
    for decl in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";"):
        if decl.strip():
            ctype, names = decl.strip().split(None, 1)
            fields += [(n.strip(), {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}[ctype]) for n in names.split(",")]
    return fields


def test_structs_match_header():
    from paper_2511_14617_amd import binding as b
    assert struct_fields("seer_reserve_params") == list(b.SeerReserveParams._fields_)
    assert struct_fields("seer_append_params") == list(b.SeerAppendParams._fields_)


def rp(**kw):
    from paper_2511_14617_amd.binding import SeerReserveParams
    base = dict(B=4, page_size=16, num_pages=100, max_pages_per_seq=32, n_tokens=50)
    base.update(kw)
    return SeerReserveParams(**base)


def test_reserve_workspace(lib):
    from paper_2511_14617_amd import binding as b
    size = b.seer_kv_reserve_workspace
    assert size(rp()) > 0 and size(rp(num_pages=1 << 20)) > 4 << 20 and size(rp(num_pages=1 << 30, page_size=1)) > 4 << 30
    for bad in (rp(B=0), rp(B=-1), rp(B=16385), rp(page_size=0), rp(num_pages=0), rp(max_pages_per_seq=0), rp(n_tokens=-1), rp(num_pages=1 << 27),
                rp(num_pages=(1 << 30) + 1, page_size=1), rp(max_pages_per_seq=1 << 27), rp(n_tokens=2 ** 31 - 1)):
        assert size(bad) == 0
    assert lib.seer_kv_reserve_workspace(None) == 0


def test_reserve_argument_errors_before_any_launch(lib):
    from paper_2511_14617_amd import binding as b

    def run(p, null=(), off=None, ws=0x10000, ws_bytes=1 << 40):
        names = ["ctx", "new", "share", "mask", "table", "held", "refs", "step", "first", "slot", "position", "status"]
        args = [None if n in null else FAKE * (i + 1) + (off[1] if off and off[0] == n else 0) for i, n in enumerate(names)]
        return lib.seer_kv_reserve(None if p is None else ctypes.byref(p), *args, ws, ws_bytes, None)

    assert run(None) == b.SEER_EINVAL
    for bad in (dict(B=-1), dict(page_size=0), dict(num_pages=0), dict(max_pages_per_seq=0), dict(n_tokens=-1)):
        assert run(rp(**bad)) == b.SEER_EINVAL, bad
    for bad in (dict(B=16385), dict(num_pages=1 << 27), dict(num_pages=(1 << 30) + 1, page_size=1), dict(max_pages_per_seq=1 << 27), dict(n_tokens=2 ** 31 - 1)):
        assert run(rp(**bad)) == b.SEER_ESHAPE, bad
    for name in ("ctx", "new", "table", "held", "refs", "step", "first", "slot", "position"):
        assert run(rp(), null=(name,)) == b.SEER_EINVAL, name
        assert run(rp(), off=(name, 2)) == b.SEER_EALIGN, name
    for name in ("share", "status"):
        assert run(rp(), off=(name, 2)) == b.SEER_EALIGN, name
    assert run(rp(), off=("mask", 4)) == b.SEER_EALIGN
    assert run(rp(), off=("refs", 4)) == b.SEER_EALIGN
    assert run(rp(), ws=None) == b.SEER_EWORKSPACE
    assert run(rp(), ws_bytes=255) == b.SEER_EWORKSPACE
    assert run(rp(num_pages=1 << 20), ws_bytes=b.seer_kv_reserve_workspace(rp(num_pages=1 << 20)) - 1) == b.SEER_EWORKSPACE
    assert run(rp(), ws=0x10004) == b.SEER_EALIGN
    # the lengths of the step and those before it are two arrays
    args = [FAKE, FAKE * 2, None, None, FAKE * 3, FAKE * 4, FAKE * 5, FAKE, FAKE * 6, FAKE * 7, FAKE * 8, None, 0x10000, 1 << 40, None]
    assert lib.seer_kv_reserve(ctypes.byref(rp()), *args) == b.SEER_EINVAL
    assert run(rp(B=0)) == b.SEER_OK


def ap(**kw):
    from paper_2511_14617_amd.binding import SeerAppendParams
    base = dict(n_tokens=10, Hq=8, Hkv=2, Dqk=128, Dv=128, page_size=16, num_pages=100, kv_shared_latent=0, rotary_at=0, rotary_dim=128, interleaved=0,
                q_stride=1024, k_stride=256, v_stride=256, q_out_stride=1024)
    base.update(kw)
    return SeerAppendParams(**base)


def test_append_argument_errors_before_any_launch(lib):
    from paper_2511_14617_amd import binding as b

    def run(p, null=(), off=None):
        names = ["q", "k", "v", "slot", "position", "inv", "q_out", "kp", "vp", "status"]
        args = [None if n in null else FAKE * (i + 1) + (off[1] if off and off[0] == n else 0) for i, n in enumerate(names)]
        return lib.seer_kv_append(None if p is None else ctypes.byref(p), *args, None)

    assert run(None) == b.SEER_EINVAL
    for bad in (dict(n_tokens=-1), dict(Hq=-1), dict(Hkv=0), dict(page_size=0), dict(num_pages=0)):
        assert run(ap(**bad)) == b.SEER_EINVAL, bad
    for bad in (dict(Dqk=0), dict(Dqk=12), dict(Dqk=4104, q_stride=1 << 20, k_stride=1 << 20, q_out_stride=1 << 20), dict(Dv=4), dict(Dv=4104, v_stride=1 << 20),
                dict(Hq=4097, q_stride=1 << 30, q_out_stride=1 << 30), dict(Hq=4096, Hkv=1, q_stride=1 << 30, q_out_stride=1 << 30),
                dict(rotary_dim=-16), dict(rotary_dim=24), dict(rotary_dim=144), dict(rotary_dim=4, interleaved=1), dict(rotary_at=8), dict(rotary_at=4, rotary_dim=64),
                dict(rotary_at=-8), dict(rotary_at=2 ** 31 - 8), dict(num_pages=1 << 27), dict(q_stride=1016), dict(k_stride=248), dict(v_stride=248), dict(q_out_stride=1016)):
        assert run(ap(**bad)) == b.SEER_ESHAPE, bad
    for bad in (dict(q_stride=1028), dict(k_stride=260), dict(v_stride=257), dict(q_out_stride=1025)):
        assert run(ap(**bad)) == b.SEER_EALIGN, bad
    for name in ("q", "k", "v", "slot", "position", "inv", "q_out", "kp", "vp"):
        assert run(ap(), null=(name,)) == b.SEER_EINVAL, name
        assert run(ap(), off=(name, 2)) == b.SEER_EALIGN, name
    assert run(ap(), off=("status", 2)) == b.SEER_EALIGN
    assert run(ap(Hq=0, q_stride=0, q_out_stride=0)) == b.SEER_EINVAL                      # (a q that no head takes)
    assert run(ap(kv_shared_latent=1)) == b.SEER_EINVAL and run(ap(kv_shared_latent=1), null=("v",)) == b.SEER_EINVAL
    assert run(ap(n_tokens=0)) == b.SEER_OK
    assert run(ap(Dqk=8, Dv=8, Hq=1, Hkv=1, rotary_dim=0, q_stride=8, k_stride=8, v_stride=8, q_out_stride=8, n_tokens=0)) == b.SEER_OK


def pp(**kw):
    from paper_2511_14617_amd.binding import SeerAttnParams
    base = dict(B=4, T=0, Hq=8, Hkv=2, Dqk=128, Dv=128, page_size=16, num_pages=100, max_pages_per_seq=32, max_splits=-7, kv_shared_latent=0, flags=-1, scale=0.088)
    base.update(kw)
    return SeerAttnParams(**base)


@pytest.mark.parametrize("heads", [(64, 8, 128, 128), (16, 16, 128, 128), (8, 1, 128, 128), (8, 1, 256, 256)])
def test_prompt_attention_workspace_of_more_tokens_does_for_fewer(lib, heads):
    from paper_2511_14617_amd import binding as b
    Hq, Hkv, Dqk, Dv = heads
    for B in (1, 2, 16, 300):
        p = b.SeerAttnParams(B, 1, Hq, Hkv, Dqk, Dv, 16, 40000, 4000, 0, 0, 0, 0.1)
        sizes = [b.seer_prompt_attention_workspace(p, n) for n in (1, 50, 1000, 1024, 1025, 2047, 2048, 2049, 8191, 8192, 16384, 16385, 40000, 500000)]
        assert sizes[0] > 0 and sizes == sorted(sizes)


def test_prompt_attention_workspace(lib):
    from paper_2511_14617_amd import binding as b
    size = b.seer_prompt_attention_workspace
    assert 0 < size(pp(), 1) <= size(pp(), 100000) <= size(pp(max_pages_per_seq=8192), 100000) < 1 << 28
    for Dqk, Dv in ((64, 64), (192, 128), (256, 256), (576, 512)):
        assert size(pp(Dqk=Dqk, Dv=Dv, kv_shared_latent=Dqk == 576), 1000) > 0
    for bad in (pp(B=0), pp(B=-1), pp(Hq=0), pp(Hkv=3), pp(Dqk=96), pp(Dv=64), pp(page_size=0), pp(num_pages=0), pp(max_pages_per_seq=0), pp(scale=0.0), pp(scale=float("nan"))):
        assert size(bad, 10) == 0
    assert size(pp(), 0) == 0 and size(pp(), -1) == 0 and lib.seer_prompt_attention_workspace(None, 5) == 0


def test_prompt_attention_argument_errors_before_any_launch(lib):
    from paper_2511_14617_amd import binding as b

    def run(p, n=50, null=(), off=None, ws=0x10000, ws_bytes=1 << 40):
        names = ["out", "q", "kp", "vp", "table", "ctx", "first"]
        args = [None if k in null else FAKE * (i + 1) + (off[1] if off and off[0] == k else 0) for i, k in enumerate(names)]
        return lib.seer_prompt_attention(*args, None if p is None else ctypes.byref(p), n, off[1] if off and off[0] == "status" else None, ws, ws_bytes, None)

    assert run(None) == b.SEER_EINVAL and run(pp(), n=-1) == b.SEER_EINVAL
    for bad in (dict(B=-1), dict(Hq=0), dict(Hkv=0), dict(page_size=0), dict(num_pages=0), dict(max_pages_per_seq=0), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("inf")), dict(scale=float("nan"))):
        assert run(pp(**bad)) == b.SEER_EINVAL, bad
    for bad in (dict(Hkv=3), dict(max_pages_per_seq=1 << 27), dict(num_pages=1 << 30, page_size=16)):
        assert run(pp(**bad)) == b.SEER_ESHAPE, bad
    assert run(pp(max_pages_per_seq=1 << 26, Hq=1 << 14, Hkv=1), n=1 << 30) == b.SEER_ESHAPE
    for bad in (dict(Dqk=96, Dv=96), dict(Dqk=128, Dv=64), dict(Dqk=576, Dv=512), dict(Dqk=576, Dv=576, kv_shared_latent=1), dict(Dqk=128, kv_shared_latent=1)):
        assert run(pp(**bad)) == b.SEER_EUNSUPPORTED, bad
    for name in ("out", "q", "kp", "vp", "table", "ctx", "first"):
        assert run(pp(), null=(name,)) == b.SEER_EINVAL, name
        assert run(pp(), off=(name, 2)) == b.SEER_EALIGN, name
    for name in ("out", "q", "kp", "vp"):
        assert run(pp(), off=(name, 8)) == b.SEER_EALIGN, name
    assert run(pp(), off=("status", 2)) == b.SEER_EALIGN
    assert run(pp(), ws=None) == b.SEER_EWORKSPACE
    assert run(pp(), ws_bytes=b.seer_prompt_attention_workspace(pp(), 50) - 1) == b.SEER_EWORKSPACE
    assert run(pp(), ws=0x10010) == b.SEER_EALIGN
    assert run(pp(B=0)) == b.SEER_OK and run(pp(), n=0) == b.SEER_OK


def test_the_binding_refuses_other_tensors():
    """On the CPU: nothing here is on a device, which is the last thing that the checks look at."""
    import torch
    from paper_2511_14617_amd import binding as b
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="n_tokens"):
        b.seer_kv_reserve(i32(2, 3), i32(2), i32(9), i32(2), i32(2), -1, 16)
    with pytest.raises(ValueError, match="page_size"):
        b.seer_kv_reserve(i32(2, 3), i32(2), i32(9), i32(2), i32(2), 5, 2 ** 32 + 16)
    with pytest.raises(ValueError, match="block_table"):
        b.seer_kv_reserve(i32(2), i32(2), i32(9), i32(2), i32(2), 5, 16)
    with pytest.raises(ValueError, match="want k "):
        b.seer_kv_append(None, bf(4, 2), None, i32(4), None, bf(3, 2, 16, 8), None)
    with pytest.raises(ValueError, match="want q "):
        b.seer_prompt_attention(bf(4, 2), bf(3, 2, 16, 64), None, i32(2, 3), i32(2), i32(3), 1.0)
    with pytest.raises(ValueError, match="Dv"):
        b.seer_prompt_attention(bf(4, 2, 576), bf(3, 1, 16, 576), None, i32(2, 3), i32(2), i32(3), 1.0)


@pytest.mark.gpu
def test_the_binding_refuses_tensors_of_other_places():
    """On the GPU machine: host tensors, other types and shapes, tensors that are not contiguous."""
    import torch
    from paper_2511_14617_amd import binding as b
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    for name, args in (("block_table", (i32(2, 3).cpu(), i32(2), i32(9), i32(2), i32(2))), ("pages_held", (i32(2, 3), i32(3), i32(9), i32(2), i32(2))),
                       ("page_refs", (i32(2, 3), i32(2), i32(18)[::2], i32(2), i32(2))), ("ctx_len", (i32(2, 3), i32(2), i32(9), i32(2).long(), i32(2))),
                       ("n_new", (i32(2, 3), i32(2), i32(9), i32(2), i32(2).cpu()))):
        with pytest.raises(ValueError, match=name):
            b.seer_kv_reserve(*args, 5, 16)
    with pytest.raises(ValueError, match="slot"):
        b.seer_kv_append(None, bf(4, 2, 8), None, i32(5), None, bf(3, 2, 16, 8), None)
    with pytest.raises(ValueError, match="k: want"):
        b.seer_kv_append(None, bf(4, 2, 8).cpu(), None, i32(4), None, bf(3, 2, 16, 8), None)
    with pytest.raises(ValueError, match="q: want"):
        b.seer_kv_append(bf(4, 2, 16), bf(4, 2, 8), None, i32(4), None, bf(3, 2, 16, 8), None)
    with pytest.raises(ValueError, match="position"):
        b.seer_kv_append(None, bf(4, 2, 8), None, i32(4), None, bf(3, 2, 16, 8), None, inv_freq=torch.ones(4, device="cuda"))
    good = (bf(4, 2, 64), bf(3, 1, 16, 64), bf(3, 1, 16, 64), i32(2, 3), i32(2), i32(3), 1.0)
    for k, name in enumerate(("q", "k_pages", "v_pages", "block_table", "ctx_len", "first_token")):
        with pytest.raises(ValueError, match=name):
            b.seer_prompt_attention(*[x.cpu() if i == k else x for i, x in enumerate(good)])
    with pytest.raises(b.SeerError, match="head"):
        b.seer_prompt_attention(bf(4, 2, 96), bf(3, 1, 16, 96), bf(3, 1, 16, 96), *good[3:])
