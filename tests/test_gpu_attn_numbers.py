"""Sparse attention whose selection holds a row that is not a number, in every form: the log-sum-exp is none, not that of an empty
row, so the probabilities worked out from it are none and no position's weight grows by them."""
import pytest
import torch

import paper_2603_12201_amd as ic

pytestmark = pytest.mark.gpu
SCALE = 1.0 / 24.0


@pytest.mark.parametrize("B, T, L, H, k, d", [
    (1, 1, 3001, 32, 2048, 576),                  # splits, few and many
    (40, 1, 2100, 32, 2048, 576),
    (64, 1, 256, 32, 64, 576),                    # a query per workgroup
    (1, 300, 400, 20, 130, 576),                  # streams of rows
    (1, 600, 2100, 17, 2048, 576),
    (1, 2300, 2300, 32, 2048, 576),               # leading rows that are whole prefixes, and the others
    (2, 1, 3001, 8, 2048, 64),                    # 64 features: splits, none
    (2, 400, 600, 8, 70, 64),
])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_log_sum_exp_of_a_row_without_numbers(B, T, L, H, k, d, bad):
    print("[case] B=%d T=%d L=%d H=%d k=%d d=%d, %g" % (B, T, L, H, k, d, bad), flush=True)
    dv, off, row = (512, 0, 576) if d == 576 else (64, 64, 128)
    g = torch.Generator().manual_seed(k + T)
    Q = torch.randn((B, T, H, d), generator=g).to(torch.bfloat16)
    Q[..., d - 2] = 1.0                                                          # (an infinity there scores +inf)
    KV = torch.randn((B, L, row), generator=g).to(torch.bfloat16)
    KV[0, 5, d - 2] = bad
    idx = torch.arange(k, dtype=torch.int32).expand(B, T, k).clone()             # causal: query t sees L - T + 1 + t positions
    idx[idx >= (L - T + 1 + torch.arange(T, dtype=torch.int32))[None, :, None]] = -1
    hit = (idx == 5).any(-1)
    hit[1:] = False
    Qd, xd = Q.cuda(), idx.cuda()
    O, lse = ic.sparse_attn(Qd, KV.cuda(), xd, dv, off, SCALE, want_lse=True)
    assert lse.cpu()[hit].isnan().all() and O.cpu()[hit].isnan().all()
    assert lse.cpu()[~hit].isfinite().all() and O.cpu()[~hit].isfinite().all()
    p = ic.attn_probs(Qd, KV.cuda(), xd, SCALE, lse)
    valid = idx >= 0
    assert p.cpu()[hit & valid.any(-1)][valid[hit]].isnan().all() and p.cpu()[~hit].isfinite().all()
    # the weights are what the other queries alone leave
    w0 = torch.rand((B, L), generator=g).cuda()
    others = torch.where(hit[..., None].cuda(), torch.zeros_like(p), p)
    w, want = torch.empty_like(w0), torch.empty_like(w0)
    ic.attn_weight_add(p, xd, w0, out=w)
    ic.attn_weight_add(others, xd, w0, out=want)
    assert torch.equal(w, want)


@pytest.mark.parametrize("B, T, L, H, k, d", [(1, 1, 3001, 32, 2048, 576), (64, 1, 256, 32, 64, 576), (1, 300, 400, 20, 130, 576), (2, 400, 600, 8, 70, 64)])
def test_log_sum_exp_of_scores_of_minus_infinity(B, T, L, H, k, d):
    """A score of -inf adds nothing: with no other score the row's log-sum-exp is -inf."""
    print("[case] B=%d T=%d L=%d H=%d k=%d d=%d, -inf" % (B, T, L, H, k, d), flush=True)
    dv, off, row = (512, 0, 576) if d == 576 else (64, 64, 128)
    g = torch.Generator().manual_seed(k)
    Q = torch.randn((B, T, H, d), generator=g).to(torch.bfloat16)
    Q[..., d - 2] = 1.0
    KV = torch.randn((B, L, row), generator=g).to(torch.bfloat16)
    KV[:, 5, d - 2] = -float("inf")
    idx = torch.full((B, T, k), -1, dtype=torch.int32)
    idx[..., 0] = 5
    _, lse = ic.sparse_attn(Q.cuda(), KV.cuda(), idx.cuda(), dv, off, SCALE, want_lse=True)
    assert bool((lse == -float("inf")).all())
