"""A selected row of the 4-bit cache that holds no numbers, whether its query is split over workgroups or not: the query's output,
log-sum-exp and probabilities are none either, its weights stay what they were, and no other query sees anything of it."""
import pytest
import torch

from tests import kv4_ref
from tests.test_gpu_kv4 import SCALE, Paged, bits, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ic():
    import paper_2603_12201_amd as m
    m.lib()
    return m


def spoil(packed, row, kind):
    if kind == "block":                                                          # exponent byte 255
        packed[row, 385] = 255
    else:                                                                        # feature 512
        packed[row, 256:258] = {"nan": (0xC0, 0x7F), "inf": (0x80, 0x7F)}[kind]


# a query of 2048 rows: 16 splits, 6, one workgroup, a wave; and 300 rows, the fewest that some counts are split from
@pytest.mark.parametrize("B, k", [(2, 2048), (40, 2048), (300, 300), (600, 200), (2, 385), (12, 1021)])
@pytest.mark.parametrize("kind", ["block", "nan", "inf"])
@pytest.mark.parametrize("page", [0, 64])
def test_a_row_without_numbers_spoils_its_query_only(ic, B, k, kind, page):
    print(f"[case] {B} queries of {k} rows, {kind}, page {page}", flush=True)
    Lk = k + 37
    pg = Paged(ic, [Lk] * B, Lk, page, seed=B, ragged=False) if page else None
    n = pg.n_rows if page else B * Lk
    few = kv4_ref.pack(bits(rows_of(B, min(n, 4096), wide=False)))
    packed = few[torch.arange(n).numpy() % few.shape[0]].copy()
    clean = torch.from_numpy(packed.copy()).cuda()
    bad = sorted({1, B - 1})                                                     # sequences with such a row, early or late among the selected
    for i, b in enumerate(bad):
        s = 3 if i == 0 else k - 2
        spoil(packed, pg.row(b, s) if page else b * Lk + s, kind)
    dirty = torch.from_numpy(packed).cuda()
    Q = torch.randn((B, 1, 32, 576), generator=torch.Generator().manual_seed(k)).to(torch.bfloat16)
    Q[..., 512] = Q[..., 512].abs().clamp_min(0.1)                               # (an infinity there scores +inf)
    Q = Q.cuda()
    idx = torch.arange(k, dtype=torch.int32, device="cuda").expand(B, 1, k).contiguous()
    w0 = torch.rand((B, Lk), generator=torch.Generator().manual_seed(1)).cuda()
    got = []
    for kv4 in (clean, dirty):
        kv4 = kv4 if page else kv4.view(B, Lk, 400)
        pc = pg.pc if page else None
        O, lse = ic.sparse_attn_kv4(Q, kv4, idx, SCALE, Lk=Lk, pc=pc, want_lse=True)
        p = ic.attn_probs_kv4(Q, kv4, idx, SCALE, lse, Lk=Lk, pc=pc)
        got.append((O, lse, p, ic.attn_weight_add(p, idx, w0, out=torch.empty_like(w0))))
    good = [b for b in range(B) if b not in bad]
    for want, have in zip(*got):
        assert torch.equal(want[good], have[good])
    O, lse, p, w = got[1]
    assert O[bad].isnan().all() and lse[bad].isnan().all() and p[bad].isnan().all()
    assert torch.equal(w[bad], w0[bad])
