"""seer_prompt_attention: what a request's neighbours, a broken key and the place of a row in memory may and may not change.  Against the softmax in 64 bits
with the tolerance of the other tests of this call."""
import numpy as np
import pytest
import torch

from test_gpu_prompt_attention import call, compare, make, plain, spoil

pytestmark = pytest.mark.gpu

EIGHT_WAVES = (64, 8, 128, 128, 16)                # (from 131 072 query rows on, 8192 and more of a KV head for a request: 256 of them a workgroup)


def alone(c, b):
    lo, hi = c["first"][b].item(), c["first"][b + 1].item()
    return dict(c, q=c["q"][lo:hi], table=c["table"][b:b + 1], ctx=c["ctx"][b:b + 1], first=torch.tensor([0, hi - lo], dtype=torch.int32)), lo, hi


@pytest.mark.parametrize("heads,new,past", [((8, 2, 128, 128, 16), [700, 1, 90, 1], [100, 4000, 0, 2500]), ((4, 4, 64, 64, 20), [1, 300, 2000], [900, 0, 5]),
                                            ((8, 1, 256, 256, 32), [150, 1, 1000], [3000, 70, 0]), ((16, 2, 192, 128, 64), [33, 1200, 1], [1, 0, 5000]),
                                            ((16, 1, 576, 512, 64), [300, 1, 40], [2000, 9000, 0]), (EIGHT_WAVES, [2100, 1030], [0, 700])])
def test_a_request_alone_and_beside_others(heads, new, past):
    """Alone its row tiles are cut elsewhere (and tiles have other sizes): the same output within the tolerance, in a batch, in the batch turned round, alone."""
    c = make(31, new, past, *heads)
    want = plain(c, 200)
    both, status = call(c)
    assert status == 0
    compare(both, want, "batch")
    order = list(range(len(new)))[::-1]
    lo, hi = c["first"][:-1].tolist(), c["first"][1:].tolist()
    turned = dict(c, q=torch.cat([c["q"][lo[b]:hi[b]] for b in order]), table=c["table"][order], ctx=c["ctx"][order],
                  first=torch.tensor(np.concatenate([[0], np.cumsum([new[b] for b in order])]), dtype=torch.int32))
    out, status = call(turned)
    assert status == 0
    at = 0
    for b in order:
        both[lo[b]:hi[b]] = out[at:at + new[b]]
        at += new[b]
    compare(both, want, "turned round")
    for b in range(len(new)):
        one, lo_b, hi_b = alone(c, b)
        out, status = call(one)
        assert status == 0
        both[lo_b:hi_b] = out
    compare(both, want, "alone")


@pytest.mark.parametrize("heads,new,past,at", [((8, 2, 128, 128, 16), [200, 70], [0, 300], [100, 340]), ((4, 4, 64, 64, 20), [500], [0], [40]), ((8, 1, 256, 256, 32), [260], [40], [45]),
                                               ((16, 2, 192, 128, 64), [300], [33], [33]), ((16, 1, 576, 512, 64), [400, 3], [0, 9000], [10, 8999]), ((5, 1, 576, 512, 20), [200], [70], [80]),
                                               (EIGHT_WAVES, [2100], [0], [300]), ((8, 2, 128, 128, 16), [1, 1], [9000, 50], [4000, 50])])
def test_tokens_that_see_a_broken_key_show_it(heads, new, past, at):
    """A NaN in a key that a token sees makes its output NaN, in tiles that all rows of a row tile see as in those at the edge; tokens before that
    position are what they are without it."""
    c = make(32, new, past, *heads)
    good, _ = call(c)
    for b, j in enumerate(at):
        spoil(c["k"], b, j, c, float("nan"))
    out, status = call(c)
    assert status == 0
    first = c["first"].tolist()
    for b, j in enumerate(at):
        sees = max(first[b], first[b] + j - past[b])
        assert torch.equal(out[first[b]:sees], good[first[b]:sees])
        assert sees < first[b + 1] and torch.isnan(out[sees:first[b + 1]].float()).all()


@pytest.mark.parametrize("heads", [(64, 8, 128, 128, 16), (64, 8, 128, 128, 20), (128, 1, 576, 512, 64)])
def test_rows_behind_4_gib(heads):
    """Queries and outputs whose bytes are counted in more than 32 bits: requests across and behind the border of 4 GiB of outputs, the rows before them left alone."""
    from paper_2511_14617_amd import binding as b
    Hq, Hkv, D, Dv, page = heads
    new = [45, 1, 30]
    c = make(33, new, [0, 200, 3], *heads)
    want = plain(c)
    dev = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    border, n = 2 ** 32 // (Hq * Dv * 2), sum(new)
    q = torch.zeros((border + 80, Hq, D), dtype=torch.bfloat16, device="cuda")
    out = torch.full((border + 80, Hq, Dv), 7.0, dtype=torch.bfloat16, device="cuda")
    for begin in (border - 20, border):
        q[begin:begin + n] = dev["q"]
        b.seer_prompt_attention(q, dev["k"], dev.get("v"), dev["table"], dev["ctx"], dev["first"] + begin, c["scale"], Dv=Dv, out=out)
        compare(out[begin:begin + n], want)
        out[begin:begin + n] = 7.0
        assert all((part == 7.0).all() for part in out.split(1 << 14))


@pytest.mark.parametrize("heads", [(16, 1, 576, 512, 64), (128, 1, 576, 512, 32), (16, 1, 576, 512, 20)])
def test_single_tokens_of_many_requests_over_the_latent(heads):
    rng = np.random.default_rng(7)
    c = make(34, [1] * 24, rng.integers(3000, 9000, 24), *heads)
    out, status = call(c)
    assert status == 0
    compare(out, plain(c))
