"""The workspace of the attention weights: kept scores only up to 2 GiB, and the same sums without them."""
import numpy as np
import pytest

GIB = 1 << 30


def params(**kw):
    from paper_2511_14617_amd.binding import SeerAttnParams
    base = dict(B=64, T=1, Hq=32, Hkv=8, Dqk=128, Dv=128, page_size=16, num_pages=100, max_pages_per_seq=8192, max_splits=0, kv_shared_latent=0, flags=0, scale=0.088)
    base.update(kw)
    return SeerAttnParams(**base)


def test_kept_scores_take_at_most_two_gib():
    from paper_2511_14617_amd import binding as b
    size = b.seer_kv_weights_workspace
    assert GIB <= size(params()) < GIB + (64 << 20)                                      # 64 x 8 x 131 072 positions of 4 scores
    assert 2 * GIB <= size(params(B=128)) < 2 * GIB + (64 << 20)                         # exactly the limit
    for kw in (dict(B=129), dict(B=128, Hq=128), dict(B=512, max_pages_per_seq=65536), dict(B=128, Hq=16, Hkv=1, Dqk=576, page_size=64, max_pages_per_seq=1 << 14),
               dict(B=1, Hq=4, Hkv=1, page_size=1024, max_pages_per_seq=(1 << 21) - 1)):
        assert 0 < size(params(**kw)) < (128 << 20), kw


@pytest.mark.gpu
@pytest.mark.parametrize("D,T,Hq,Hkv,P", [(128, 4, 16, 4, 16), (64, 2, 12, 3, 20), (576, 1, 16, 1, 64)])
def test_few_rows_on_tables_beyond_the_limit(D, T, Hq, Hkv, P):
    """Two sweeps for 16, 8 and 16 rows, on a table with thousands of positions that no request has."""
    import torch
    from paper_2511_14617_amd import binding
    from test_gpu_kv_weights import build, reference
    s = build(3, T, Hq, Hkv, D, P, [700, T, 1300], D, T > 1)
    want, tol = reference(s, 0.75)
    kept = 8 if D == 64 else 16
    pages = 2 * GIB // (4 * kept * 3 * Hkv * P) + 1
    table = torch.full((3, pages), 1 << 30, dtype=torch.int32, device="cuda")
    table[:, :s["table"].shape[1]] = s["table"]
    w = torch.full((3, Hkv, pages * P), 5.0, device="cuda")
    n = s["w"].shape[2]
    w[:, :, :n] = s["w"]
    p = binding.attn_params(s["q"], s["k"], None, table, s["scale"], Dv=D)
    assert binding.seer_kv_weights_workspace(p) < (64 << 20)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.seer_kv_weights(w, s["q"], s["k"], table, s["ctx"], s["alen"], s["path"], s["scale"], decay=0.75, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0 and (w[:, :, n:] == 5).all()
    assert (np.abs(w[:, :, :n].double().cpu().numpy() - want) <= tol).all()
