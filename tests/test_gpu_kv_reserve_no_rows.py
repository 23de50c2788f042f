"""seer_kv_reserve for a step without rows: there is nothing to reserve, and every token of the call is padding."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def i32(*shape, fill=0):
    return torch.full(shape, fill, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n_tokens,pages", [(0, 10), (1, 10), (50, 10), (9000, 40000)])
@pytest.mark.parametrize("given", [False, True])
def test_all_tokens_are_padding(n_tokens, pages, given):
    from paper_2511_14617_amd import binding as b
    junk = [i32(2 * n_tokens + 100, fill=5) for _ in range(4)]           # (what new memory of this size holds behind it)
    torch.cuda.synchronize()
    del junk
    out = (i32(0), i32(1, fill=5), i32(n_tokens, fill=5), i32(n_tokens, fill=5)) if given else None
    refs, status = i32(pages, fill=1), i32(1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for s in (None, stream):
        step_len, first_token, slot, position = b.seer_kv_reserve(i32(0, 4), i32(0), refs, i32(0), i32(0), n_tokens, 16, out=out, status=status, stream=s)
        torch.cuda.synchronize()
        assert step_len.numel() == 0 and first_token.tolist() == [0]
        assert slot.tolist() == [-1] * n_tokens and position.tolist() == [-1] * n_tokens
        if given:
            for x in out:
                x.fill_(5)
    assert status.item() == 0 and (refs == 1).all()


def test_no_row_reaches_the_cache():
    """The rows of a step without requests, appended: no slot, so nothing is written."""
    from paper_2511_14617_amd import binding as b
    junk = i32(200, fill=3)
    torch.cuda.synchronize()
    del junk
    made = b.seer_kv_reserve(i32(0, 4), i32(0), i32(10), i32(0), i32(0), 90, 16)
    k = torch.ones((90, 2, 64), dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros((10, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    b.seer_kv_append(None, k, None, made[2], made[3], pool, None, inv_freq=torch.ones(32, device="cuda"))
    assert not pool.any()


def test_captured():
    from paper_2511_14617_amd import binding as b
    out, refs = (i32(0), i32(1), i32(40), i32(40)), i32(10)
    table, rows, ws = i32(0, 4), i32(0), torch.empty(256, dtype=torch.uint8, device="cuda")
    call = lambda: b.seer_kv_reserve(table, rows, refs, rows, rows, 40, 16, out=out, workspace=ws)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for x in out:
            x.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert out[1].tolist() == [0] and out[2].tolist() == out[3].tolist() == [-1] * 40
