"""A selected row of the 4-bit cache that holds no numbers, whether its query is split over workgroups or not: the query's output,
log-sum-exp and probabilities are none either, its weights stay what they were, and no other query sees anything of it."""
import numpy as np
import pytest
import torch

from tests import kv4_ref
from tests.test_gpu_kv4 import SCALE, Paged, bits, check_query, rows_of

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


# few queries, a wave each with the weights four waves to a query, and a wave each for both
@pytest.mark.parametrize("T", [2, 600, 800])
@pytest.mark.parametrize("paged", [False, True])
def test_rows_on_both_sides_of_4_gib(ic, T, paged):
    """11.2 million rows: some in front of the first that begins behind 4 GiB, some around it, some at the end."""
    n = 175000 * 64
    first = -(-(1 << 32) // 400)
    print(f"[case] {T} queries over {n} rows, paged {paged}", flush=True)
    kv4 = torch.empty((n, 400), dtype=torch.uint8, device="cuda")
    x = rows_of(14, 192, wide=False)
    at = [0, first - first % 64, n - 64]
    if paged:
        Lk, pc = 192, ic.paged_cache(None, torch.tensor([[a // 64 for a in at]], dtype=torch.int32, device="cuda"), 64)
        pos = np.arange(192)
        ic.kv4_write(x.cuda()[None], kv4, Lk=Lk, pc=pc)
    else:
        Lk, pc = n, None
        kv4 = kv4[None]
        pos = np.concatenate([np.arange(a, a + 64) for a in at])
        for i, a in enumerate(at):
            ic.kv4_write(x[64 * i:64 * i + 64].cuda()[None], kv4, pos0=a)
    want = kv4_ref.pack(bits(x))
    for i, a in enumerate(at):
        assert np.array_equal(kv4.view(n, 400)[a:a + 64].cpu().numpy(), want[64 * i:64 * i + 64])
    Q = torch.randn((1, T, 32, 576), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    sel = np.stack([np.sort(np.random.default_rng(t).permutation(192)[:150]) for t in range(T)])
    idx = torch.from_numpy(pos[sel].astype(np.int32)).cuda()[None]
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, idx, SCALE, Lk=Lk, pc=pc, want_lse=True)
    probs = ic.attn_probs_kv4(Q.cuda(), kv4, idx, SCALE, lse, Lk=Lk, pc=pc)
    rows, Qf = kv4_ref.unpack(want), kv4_ref.bf16_bits_to_f64(bits(Q))
    for t in sorted({0, 1, T // 2, T - 1}):
        check_query(O[0, t], lse[0, t], probs[0, t], Qf[0, t], rows[sel[t]], np.ones(150, dtype=bool))


@pytest.mark.parametrize("T, k", [(1, 40), (1, 700), (40, 2048), (300, 300), (700, 200)])
@pytest.mark.parametrize("power", [20, 25, 26, 27, 28, 29, 30, 31, 40, 90])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(ic, T, k, power, sign):
    """One feature decides: row r scores sign (1 + r / 64 % 1) 2^power, exactly, so that equal rows share the weight and it is their mean."""
    print(f"[case] {T} queries of {k} rows, scores about {sign} 2^{power}", flush=True)
    x = rows_of(17, k, wide=False)
    x[:, 512:] = 0
    step = torch.arange(k) * 7 % 64
    x[:, 512] = sign * (1 + step / 64.0) * 2.0 ** (power // 2)
    Q = torch.zeros((1, T, 32, 576), dtype=torch.bfloat16)
    Q[..., 512] = 2.0 ** (power - power // 2)
    kv4 = torch.empty((1, k, 400), dtype=torch.uint8, device="cuda")
    ic.kv4_write(x.cuda()[None], kv4)
    idx = torch.arange(k, dtype=torch.int32, device="cuda").expand(1, T, k).contiguous()
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, idx, 1.0, want_lse=True)
    top = int(step.max() if sign > 0 else step.min())
    rows = kv4_ref.unpack(kv4.cpu().numpy()[0])[(step == top).numpy()]
    want = rows[:, :512].mean(0)
    # weights 1 / n in bf16, 2^-8 each, and the output's 2^-8; the next lower scores are 2^(power - 6) further down
    tol = 2.0 ** -8 * np.abs(rows[:, :512]).mean(0) + 2.0 ** -8 * np.abs(want) + 2.0 ** -20
    assert np.all(np.abs(O[0].double().cpu().numpy() - want) <= tol)
    l = sign * (1 + top / 64.0) * 2.0 ** power + np.log(len(rows))
    assert np.all(np.abs(lse.double().cpu().numpy() - l) <= 2.0 ** -20 * (1 + abs(l)))


@pytest.mark.parametrize("B, k", [(2, 2048), (40, 2048), (300, 300), (600, 200)])
def test_a_score_of_minus_infinity_is_a_skipped_entry(ic, B, k):
    print(f"[case] {B} queries of {k} rows, -inf", flush=True)
    packed = kv4_ref.pack(bits(rows_of(B, k, wide=False)))
    gone = [0, 5, k // 2, k - 1] + list(range(64, 128))                          # (whole tiles among them)
    packed[gone, 256:258] = (0x80, 0xFF)
    kv4 = torch.from_numpy(packed).cuda()[None].expand(B, k, 400).contiguous()
    Q = torch.randn((B, 1, 32, 576), generator=torch.Generator().manual_seed(k)).to(torch.bfloat16)
    Q[..., 512] = Q[..., 512].abs().clamp_min(0.1)
    idx = torch.arange(k, dtype=torch.int32, device="cuda").expand(B, 1, k).contiguous()
    skip = idx.clone()
    skip[..., gone] = -1
    got, want = [ic.sparse_attn_kv4(Q.cuda(), kv4, i, SCALE, want_lse=True) for i in (idx, skip)]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    p, q = [ic.attn_probs_kv4(Q.cuda(), kv4, i, SCALE, want[1]) for i in (idx, skip)]
    assert torch.equal(p, q)
    only = torch.full_like(idx, -1)                                              # nothing but such rows
    only[..., gone] = idx[..., gone]
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, only, SCALE, want_lse=True)
    assert not O.any() and bool((lse == -float("inf")).all())
