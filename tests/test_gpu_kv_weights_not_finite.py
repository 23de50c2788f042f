"""Attention weights with queries and keys that are not finite: a NaN among the scores of a row makes the weight of every position that the row sees a NaN,
on every path and wherever the request is cut, and leaves what the row does not see alone."""
import pytest
import torch

from test_gpu_kv_weights import build

pytestmark = pytest.mark.gpu

# one kernel for short tables, kept scores, two sweeps with one wave (from three, from one row on) and with two, the shared latent with kept scores and with eight waves
PATHS = {
    "short": dict(Hq=8, Hkv=2, D=128, P=16, extra_pages=0),
    "kept": dict(Hq=8, Hkv=2, D=128, P=16, extra_pages=40),
    "one wave": dict(Hq=12, Hkv=2, D=256, P=32, extra_pages=40),
    "two sweeps": dict(Hq=40, Hkv=2, D=128, P=16, extra_pages=40),
    "two waves": dict(Hq=80, Hkv=2, D=64, P=20, extra_pages=40),
    "latent kept": dict(Hq=6, Hkv=2, D=576, P=64, extra_pages=10),
    "latent": dict(Hq=128, Hkv=1, D=576, P=64, extra_pages=10),
}
EVERY = pytest.mark.parametrize("path", sorted(PATHS))


def setup(path, T, ctx, seed, **kw):
    d = dict(PATHS[path], **kw)
    return build(len(ctx), T, d["Hq"], d["Hkv"], d["D"], d["P"], ctx, seed, extra_pages=d["extra_pages"])


def run(s, decay=1.0):
    from paper_2511_14617_amd import binding
    w, status = s["w"].clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.seer_kv_weights(w, s["q"], s["k"], s["table"], s["ctx"], s["alen"], s["path"], s["scale"], decay=decay, status=status)
    assert status.item() == 0
    return w


@EVERY
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite(path, bad):
    """The last row of a step sees everything: its head group is NaN throughout, nothing else changes.  (An infinite query gives infinities of both signs.)"""
    s = setup(path, 4, [200, 150], 1)
    clean = run(s)
    s["q"][0, 3, 0, 5] = bad
    w = run(s)
    assert torch.isnan(w[0, 0, :200]).all()
    assert torch.equal(w[1], clean[1]) and torch.equal(w[0, 1:], clean[0, 1:]) and torch.equal(w[0, 0, 200:], clean[0, 0, 200:])


@EVERY
def test_a_key_that_is_alone_in_its_tile(path):
    """Positions 32 i of a request of 32 i + 1: the only one of its tile, and of its piece where the request is cut there."""
    lengths = [225, 193, 33, 161]
    s = setup(path, 1, lengths, 2)
    clean = run(s)
    page = PATHS[path]["P"]
    at = lengths[0] - 1
    s["k"][s["table"][0, at // page].long(), 0, at % page, 3] = float("nan")
    w = run(s)
    assert torch.isnan(w[0, 0, :225]).all()
    assert torch.equal(w[1:], clean[1:]) and torch.equal(w[0, 1:], clean[0, 1:])


@pytest.mark.parametrize("path", ["kept", "two sweeps", "two waves", "latent"])
@pytest.mark.parametrize("where", [(0, 2000), (2048, 4096), (3, 4), (5998, 6000)])
def test_a_stretch_of_keys(path, where):
    """NaN keys that fill whole pieces, at the beginning, inside and at the end."""
    s = setup(path, 1, [6000, 3000], 3)
    clean = run(s)
    page = PATHS[path]["P"]
    pos = torch.arange(*where, device="cuda")
    s["k"][s["table"][0, pos // page].long(), 0, pos % page] = float("nan")
    w = run(s)
    assert torch.isnan(w[0, 0, :6000]).all()
    assert torch.equal(w[1], clean[1]) and torch.equal(w[0, 1:], clean[0, 1:])
