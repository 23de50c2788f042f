"""seer_prompt_attention with block tables that have room for far longer requests than there are.  Against the softmax in 64 bits with the tolerance of the other
tests of this call."""
import pytest
import torch

from test_gpu_prompt_attention import call, compare, make, plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(8, 1, 128, 128, 16), (8, 2, 64, 64, 20), (4, 1, 256, 256, 16), (16, 2, 192, 128, 16), (16, 1, 576, 512, 64)])
@pytest.mark.parametrize("new,past", [([1] * 16, [4096] * 16), ([1, 40, 300, 2], [700, 0, 20, 3000]), ([1], [0])])
def test_block_tables_much_wider_than_the_contexts(heads, new, past):
    """A server's tables have room for the longest request: most workgroups of the launch have nothing to do, and none of the rest's results is theirs.  Twice in one
    workspace that held something else."""
    c = make(35, new, past, *heads)
    c["table"] = torch.nn.functional.pad(c["table"], (0, 131072 // c["page"]), value=-9)
    want = plain(c)
    from paper_2511_14617_amd import binding as b
    p = b.attn_params(c["q"].unsqueeze(1), c["k"], c["v"], c["table"], c["scale"], c["Dv"])
    p.B = len(new)
    ws = torch.full((b.seer_prompt_attention_workspace(p, sum(new)),), 0x77, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        out, status = call(c, workspace=ws)
        assert status == 0
        compare(out, want)
    empty = dict(c, first=torch.zeros_like(c["first"]))
    out, status = call(empty, workspace=ws)
    assert status == 0 and (out == 7.0).all()
