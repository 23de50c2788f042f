"""Host-side checks, without a GPU, of the calls that record log probabilities and keep the cache small: parameter structs,
workspace sizes, and bad arguments turned into SEER_E* codes before anything is launched."""
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


def lp(**kw):
    from paper_2511_14617_amd.binding import SeerLogprobParams
    base = dict(B=4, T=5, V=1000, ld=1000, dtype=0, top_n=3, temperature=1.0)
    base.update(kw)
    return SeerLogprobParams(**base)


def test_logprob_struct_matches_header():
    from paper_2511_14617_amd.binding import SeerLogprobParams
    assert struct_fields("seer_logprob_params") == list(SeerLogprobParams._fields_)


def test_logprob_workspace(lib):
    from paper_2511_14617_amd import binding as b
    size = b.seer_token_logprobs_workspace
    assert size(lp()) > 0 and size(lp()) % 256 == 0
    assert size(lp(V=152064, ld=152064)) > size(lp()) and size(lp(top_n=32)) > size(lp(top_n=0)) > 0
    for bad in (lp(B=0), lp(B=-1), lp(T=0), lp(V=0), lp(ld=999), lp(top_n=33), lp(top_n=-1), lp(V=2, ld=2), lp(dtype=2), lp(temperature=0.0)):
        assert size(bad) == 0
    assert lib.seer_token_logprobs_workspace(None) == 0


def test_logprob_argument_errors_before_any_launch(lib):
    from paper_2511_14617_amd import binding as b

    def run(p, logits=FAKE, tokens=FAKE, path=None, out=FAKE, ent=None, top=FAKE, topi=FAKE, ws=0x10000, ws_bytes=1 << 40):
        return lib.seer_token_logprobs(logits, tokens, path, None if p is None else ctypes.byref(p), out, ent, None, top, topi, ws, ws_bytes, None)

    assert run(None) == b.SEER_EINVAL
    assert run(lp(B=-1)) == b.SEER_EINVAL
    assert run(lp(V=0)) == b.SEER_EINVAL
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert run(lp(temperature=t)) == b.SEER_EINVAL, t
    for bad in (dict(T=0), dict(ld=999), dict(top_n=-1), dict(top_n=33), dict(V=2, ld=2), dict(B=1 << 20, T=1 << 12),
                dict(B=1 << 30, T=1, V=1 << 20, ld=1 << 20)):
        assert run(lp(**bad)) == b.SEER_ESHAPE, bad
    assert run(lp(dtype=2)) == b.SEER_EUNSUPPORTED
    assert run(lp(V=(1 << 24) + 1, ld=1 << 25)) == b.SEER_EUNSUPPORTED
    assert run(lp(), logits=None) == b.SEER_EINVAL
    assert run(lp(), tokens=None) == b.SEER_EINVAL
    assert run(lp(), out=None) == b.SEER_EINVAL
    assert run(lp(), top=None) == b.SEER_EINVAL
    assert run(lp(), topi=None) == b.SEER_EINVAL
    assert run(lp(), ws=None) == b.SEER_EWORKSPACE
    assert run(lp(), ws_bytes=b.seer_token_logprobs_workspace(lp()) - 1) == b.SEER_EWORKSPACE
    assert run(lp(), logits=FAKE + 2) == b.SEER_EALIGN
    assert run(lp(dtype=1), logits=FAKE + 1) == b.SEER_EALIGN
    assert run(lp(), ws=0x10004) == b.SEER_EALIGN
    assert run(lp(), ent=FAKE + 2) == b.SEER_EALIGN
    assert run(lp(B=0)) == b.SEER_OK


def test_logprob_grad_argument_errors_before_any_launch(lib):
    from paper_2511_14617_amd import binding as b

    def run(p, grad=2 * FAKE, ld=1000, logits=FAKE, tokens=FAKE, lse=FAKE, ent=None, g=FAKE, gh=None):
        return lib.seer_token_logprobs_grad(grad, ld, logits, tokens, lse, ent, g, gh, None if p is None else ctypes.byref(p), None)

    assert run(None) == b.SEER_EINVAL
    assert run(lp(), ld=999) == b.SEER_ESHAPE
    assert run(lp(), grad=None) == b.SEER_EINVAL
    assert run(lp(), lse=None) == b.SEER_EINVAL
    assert run(lp(), tokens=None) == b.SEER_EINVAL
    assert run(lp(), gh=FAKE) == b.SEER_EINVAL                    # the entropy's gradient needs the entropy
    assert run(lp(), grad=FAKE, ld=1001) == b.SEER_EINVAL         # in place with other rows
    assert run(lp(), grad=FAKE + 2) == b.SEER_EALIGN
    assert run(lp(), g=FAKE + 1) == b.SEER_EALIGN
    assert run(lp(temperature=-1.0)) == b.SEER_EINVAL
    assert run(lp(B=0)) == b.SEER_OK


def attn(**kw):
    from paper_2511_14617_amd.binding import SeerAttnParams
    base = dict(B=4, T=5, Hq=8, Hkv=2, Dqk=128, Dv=128, page_size=16, num_pages=100, max_pages_per_seq=32, max_splits=0,
                kv_shared_latent=0, flags=0, scale=0.088)
    base.update(kw)
    return SeerAttnParams(**base)


def test_kv_weights_workspace_and_argument_errors_before_any_launch(lib):
    from paper_2511_14617_amd import binding as b
    size = b.seer_kv_weights_workspace
    assert size(attn()) > 0 and size(attn()) % 256 == 0
    assert size(attn(Dqk=576, Hq=128, Hkv=1, page_size=64)) > 0

    def run(p, w=FAKE, q=FAKE, k=FAKE, table=FAKE, ctx=FAKE, alen=FAKE, path=FAKE, decay=1.0, status=None, ws=0x10000, ws_bytes=1 << 40):
        return lib.seer_kv_weights(w, q, k, table, ctx, alen, path, decay, None if p is None else ctypes.byref(p), status, ws, ws_bytes, None)

    for bad, code in ((dict(B=-1), b.SEER_EINVAL), (dict(num_pages=0), b.SEER_EINVAL), (dict(scale=0.0), b.SEER_EINVAL), (dict(scale=float("nan")), b.SEER_EINVAL),
                      (dict(scale=float("inf")), b.SEER_EINVAL), (dict(T=0), b.SEER_ESHAPE), (dict(T=65), b.SEER_ESHAPE), (dict(Hq=7), b.SEER_ESHAPE),
                      (dict(Dqk=100), b.SEER_EUNSUPPORTED), (dict(page_size=0), b.SEER_EINVAL), (dict(max_pages_per_seq=1 << 30), b.SEER_ESHAPE),
                      (dict(B=1 << 20, max_pages_per_seq=1 << 16), b.SEER_ESHAPE), (dict(num_pages=1 << 30), b.SEER_ESHAPE)):
        assert run(attn(**bad)) == code, bad
        assert size(attn(**bad)) == 0, bad
    assert run(None) == b.SEER_EINVAL
    for d in (-0.1, 1.5, float("nan")):
        assert run(attn(), decay=d) == b.SEER_EINVAL
    for name in ("w", "q", "k", "table", "ctx", "alen", "path"):
        assert run(attn(), **{name: None}) == b.SEER_EINVAL, name       # (accepted_len and accepted_path come together)
    assert run(attn(), ws=None) == b.SEER_EWORKSPACE
    assert run(attn(), ws_bytes=size(attn()) - 1) == b.SEER_EWORKSPACE
    assert run(attn(), ws=0x10010) == b.SEER_EALIGN
    assert run(attn(), q=FAKE + 2) == b.SEER_EALIGN
    assert run(attn(), w=FAKE + 2) == b.SEER_EALIGN
    assert run(attn(), status=FAKE + 1) == b.SEER_EALIGN
    assert run(attn(B=0)) == b.SEER_OK


def ev(**kw):
    from paper_2511_14617_amd.binding import SeerEvictParams
    base = dict(limit=300, budget=256, keep_first=16, keep_last=32)
    base.update(kw)
    return SeerEvictParams(**base)


def test_evict_struct_matches_header():
    from paper_2511_14617_amd.binding import SeerEvictParams
    assert struct_fields("seer_evict_params") == list(SeerEvictParams._fields_)


def test_kv_evict_workspace_and_argument_errors_before_any_launch(lib):
    from paper_2511_14617_amd import binding as b
    size = b.seer_kv_evict_workspace
    assert size(attn(), ev()) > 0 and size(attn(), ev()) % 256 == 0
    assert size(attn(max_pages_per_seq=2), ev()) > 0             # a budget beyond the block table: nothing is ever cut

    def run(p, e, k=FAKE, v=FAKE, table=FAKE, ctx=FAKE, first=None, w=FAKE, new=FAKE, neww=None, kept=None, status=None, ws=0x10000, ws_bytes=1 << 40):
        return lib.seer_kv_evict(None if p is None else ctypes.byref(p), None if e is None else ctypes.byref(e), k, v, table, ctx, first, w, new, neww, kept,
                                 status, ws, ws_bytes, None)

    assert run(None, ev()) == b.SEER_EINVAL
    assert run(attn(), None) == b.SEER_EINVAL
    for bad, code in ((dict(B=-1), b.SEER_EINVAL), (dict(num_pages=0), b.SEER_EINVAL), (dict(Hkv=0), b.SEER_ESHAPE), (dict(Dqk=100), b.SEER_ESHAPE),
                      (dict(Dv=4), b.SEER_ESHAPE), (dict(Dv=0), b.SEER_ESHAPE), (dict(max_pages_per_seq=1 << 30), b.SEER_ESHAPE),
                      (dict(B=1 << 20), b.SEER_ESHAPE)):
        assert run(attn(**bad), ev()) == code, bad
        assert size(attn(**bad), ev()) == 0, bad
    for bad, code in ((dict(budget=0), b.SEER_EINVAL), (dict(limit=255), b.SEER_EINVAL), (dict(keep_first=-1), b.SEER_EINVAL), (dict(keep_last=-1), b.SEER_EINVAL),
                      (dict(keep_first=225), b.SEER_ESHAPE)):
        assert run(attn(), ev(**bad)) == code, bad
        assert size(attn(), ev(**bad)) == 0, bad
    for name in ("k", "v", "table", "ctx", "w", "new"):
        assert run(attn(), ev(), **{name: None}) == b.SEER_EINVAL, name
    assert run(attn(kv_shared_latent=1), ev()) == b.SEER_EINVAL          # the shared latent has no v_pages
    assert run(attn(), ev(), ws=None) == b.SEER_EWORKSPACE
    assert run(attn(), ev(), ws_bytes=size(attn(), ev()) - 1) == b.SEER_EWORKSPACE
    assert run(attn(), ev(), ws=0x10008) == b.SEER_EALIGN
    assert run(attn(), ev(), k=FAKE + 8) == b.SEER_EALIGN
    assert run(attn(), ev(), w=FAKE + 2) == b.SEER_EALIGN
    assert run(attn(B=0), ev()) == b.SEER_OK


def test_tensors_and_streams_of_another_device_are_refused(monkeypatch):
    import torch
    from paper_2511_14617_amd import binding as b

    class On:
        def __init__(self, i):
            self.device, self.device_index = "cuda:%d" % i, i

        def get_device(self):
            return self.device_index

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    b._here(None, logits=On(1), tokens=On(1), out=None)
    b._here(On(1), logits=On(1))
    with pytest.raises(ValueError, match="tokens: want it on the current device, cuda:1, got cuda:0"):
        b._here(None, logits=On(1), tokens=On(0))
    with pytest.raises(ValueError, match="stream"):
        b._here(On(0), logits=On(1))


@pytest.mark.parametrize("name", ["seer_token_logprobs", "seer_token_logprobs_grad", "seer_kv_weights", "seer_kv_evict"])
def test_every_tensor_of_a_call_is_looked_at(name):
    """Each tensor argument of the call, and each tensor that it makes, stands in its check of devices."""
    import inspect
    from paper_2511_14617_amd import binding as b
    source = inspect.getsource(getattr(b, name))
    looked = source[source.index("    _here("):source.index("    _check(lib." + name)]
    named = {n for n, a in inspect.signature(getattr(b, name)).parameters.items() if "Tensor" in str(a.annotation) and "Tuple" not in str(a.annotation)}
    assert named and all(re.search(r"\b%s=" % n, looked) for n in named), named
    assert "torch.empty(" not in source


def test_launches_that_a_device_cannot_count_are_refused(lib):
    """2^32 threads or more in one launch: refused on the host, below that the call has a workspace."""
    from paper_2511_14617_amd import binding as b
    lps, kvw, kve = b.seer_token_logprobs_workspace, b.seer_kv_weights_workspace, b.seer_kv_evict_workspace
    rows = (2 ** 32 - 1) // 256
    assert lps(lp(B=rows, T=1, V=100, ld=100)) > 0 and lps(lp(B=rows + 1, T=1, V=100, ld=100)) == 0
    assert lps(lp(B=rows // 2, T=1, V=20000, ld=20000)) > 0 and lps(lp(B=rows // 2 + 1, T=1, V=20000, ld=20000)) == 0
    heads = rows - 8192
    one = dict(T=1, Hq=1, Hkv=1, max_pages_per_seq=1)
    assert kvw(attn(B=heads, **one)) > 0 and kvw(attn(B=heads + 1, **one)) == 0
    assert kvw(attn(B=heads // 2, T=16, Hq=1, Hkv=1, max_pages_per_seq=1)) > 0 and kvw(attn(B=heads // 2 + 1, T=16, Hq=1, Hkv=1, max_pages_per_seq=1)) == 0
    assert kve(attn(B=(1 << 19) - 1, **one), ev()) > 0 and kve(attn(B=1 << 19, **one), ev()) == 0
    wide = dict(one, Dqk=8192, Dv=8192)                                                                     # 257 columns of 128 bytes, one workgroup more
    assert kve(attn(B=heads // 258, **wide), ev()) > 0 and kve(attn(B=heads // 258 + 1, **wide), ev()) == 0
    assert kve(attn(B=heads // 258 + 1, **wide), ev(keep_last=0)) > 0
    long = dict(one, max_pages_per_seq=1 << 14)                                                             # 64 segments and one
    assert kve(attn(B=heads // 65, **long), ev(keep_last=0)) > 0 and kve(attn(B=heads // 65 + 1, **long), ev(keep_last=0)) == 0
