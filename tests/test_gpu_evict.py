"""Eviction on the GPU: accumulated weights, the positions that stay, rows moved; and the calls together as a server makes them.

Weights: each probability is taken to 2^-48 (down), the sum is rounded to fp32 once: |dw| <= n 2^-48 + 2^-24 |w| for n entries."""
import sys

import numpy as np
import pytest
import torch

from tests import kv4_ref
from tests.test_gpu_kv4 import SCALE, Paged, bits, check_query, rows_of

pytestmark = pytest.mark.gpu


def say(msg):
    print("[case] " + msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def ic():
    import paper_2603_12201_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("B, Tq, k, Lk", [(1, 1, 1, 1), (3, 1, 100, 77), (2, 5, 64, 20000), (1, 70, 33, 50), (2, 700, 256, 900), (1, 300, 2048, 40000),
                                          (40, 1, 2048, 5000), (1, 33000, 4, 9)])
def test_weights_are_the_exact_sums(ic, B, Tq, k, Lk):
    say("weights B=%d Tq=%d k=%d Lk=%d" % (B, Tq, k, Lk))
    rng = np.random.default_rng(Tq + k)
    idx = rng.integers(-2, Lk + 2, (B, Tq, k)).astype(np.int32)                  # entries outside, and equal ones in a row
    idx[rng.random(idx.shape) < 0.01] = -(1 << 31)
    p = (rng.random((B, Tq, k)) ** 8).astype(np.float32)
    w0 = (rng.random((B, Lk)) * 10).astype(np.float32)
    want, n = w0.astype(np.float64), np.zeros((B, Lk))
    for b in range(B):
        ok = (idx[b] >= 0) & (idx[b] < Lk)
        np.add.at(want[b], idx[b][ok], p[b][ok].astype(np.float64))
        np.add.at(n[b], idx[b][ok], 1)
    pd, xd, wd = torch.from_numpy(p).cuda(), torch.from_numpy(idx).cuda(), torch.from_numpy(w0).cuda()
    out = ic.attn_weight_add(pd, xd, wd, out=torch.full_like(wd, 7.0))
    assert torch.equal(wd.cpu(), torch.from_numpy(w0))
    got = out.cpu().double().numpy()
    assert np.all(np.abs(got - want) <= n * 2.0 ** -48 + 2.0 ** -24 * np.abs(want))
    # in another order of the rows, in place: the same bits
    perm = torch.randperm(Tq, generator=torch.Generator().manual_seed(1)).cuda()
    ic.attn_weight_add(pd[:, perm].contiguous(), xd[:, perm].contiguous(), wd)
    assert torch.equal(wd, out)


def test_probabilities_outside_their_range_are_held_to_it(ic):
    p = torch.tensor([[[float("nan"), -1.0, 2.0, float("inf"), 1.0, 0.25, 1e-30, -0.0]]], device="cuda")
    idx = torch.arange(8, dtype=torch.int32, device="cuda").reshape(1, 1, 8)
    w = ic.attn_weight_add(p, idx, torch.zeros((1, 8), device="cuda"))
    assert w.cpu().tolist() == [[0.0, 0.0, 1.0, 1.0, 1.0, 0.25, 0.0, 0.0]]


def _keep_ref(w, n, n_keep, first, recent):
    if n <= n_keep:
        return list(range(n))
    inner = range(first, n - recent)
    key = lambda s: (0 if np.isnan(w[s]) else 1, -w[s] if not np.isnan(w[s]) else 0.0, s)
    best = sorted(inner, key=key)[:n_keep - first - recent]
    return sorted(list(range(first)) + best + list(range(n - recent, n)))


@pytest.mark.parametrize("Lk, n_keep, first, recent", [(1, 1, 0, 0), (5, 3, 1, 1), (100, 100, 0, 0), (1000, 999, 4, 64), (1000, 1, 0, 0), (777, 100, 100, 0),
                                                       (777, 100, 0, 100), (5000, 2500, 4, 128), (12001, 5000, 4, 64), (20011, 9000, 4, 512), (40000, 8000, 4, 512), (70001, 35000, 0, 0)])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_what_stays(ic, Lk, n_keep, first, recent, kind):
    say("evict Lk=%d keep=%d first=%d recent=%d %s" % (Lk, n_keep, first, recent, kind))
    rng = np.random.default_rng(Lk + n_keep)
    lens = [Lk, max(Lk // 2, 1), 0, 1, min(n_keep, Lk), min(n_keep + 1, Lk), Lk]
    B = len(lens)
    if kind == "spread":
        w = rng.lognormal(0, 3, (B, Lk)).astype(np.float32)
        w[0, rng.random(Lk) < 0.4] = 0
    else:
        w = rng.integers(0, 3, (B, Lk)).astype(np.float32) - 1
        w[0] = 0.5                                                               # all the same: the lowest positions
        w[1, ::2] = -0.0
        w[5, rng.random(Lk) < 0.1] = np.inf
        w[5, rng.random(Lk) < 0.1] = -np.inf
        w[6, rng.random(Lk) < 0.1] = np.nan
        w[6, rng.random(Lk) < 0.1] = -np.nan
    keep, n, kept = ic.evict_keep(torch.from_numpy(w).cuda(), n_keep, first, recent, seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    keep, n, kept = keep.cpu().numpy(), n.cpu().numpy(), kept.cpu().numpy()
    for b in range(B):
        want = _keep_ref(w[b], lens[b], n_keep, first, recent)
        assert n[b] == len(want)
        assert np.array_equal(keep[b, :n[b]], want), (b, lens[b])
        assert (keep[b, n[b]:] == -1).all() and not kept[b, n[b]:].any()
        assert np.array_equal(kept[b, :n[b]], w[b][want], equal_nan=True)
    # no lengths: every sequence has Lk
    k2, n2, _ = ic.evict_keep(torch.from_numpy(w[:1]).cuda(), n_keep, first, recent)
    assert np.array_equal(k2.cpu().numpy()[0], keep[0]) and int(n2[0]) == n[0]


def test_many_long_sequences(ic):
    """90 of 17001 positions: more parts than compute units, so a workgroup each."""
    say("evict 90 sequences of 17001")
    rng = np.random.default_rng(11)
    B, L, nk = 90, 17001, 6000
    w = rng.integers(0, 40, (B, L)).astype(np.float32)
    lens = rng.integers(1, L + 1, B).astype(np.int32)
    lens[:2] = L, nk + 1
    keep, n, kept = ic.evict_keep(torch.from_numpy(w).cuda(), nk, 8, 100, seq_lens=torch.from_numpy(lens).cuda())
    keep, n, kept = keep.cpu().numpy(), n.cpu().numpy(), kept.cpu().numpy()
    for b in range(B):
        want = np.array(_keep_ref(w[b], int(lens[b]), nk, 8, 100))
        assert n[b] == len(want) and np.array_equal(keep[b, :n[b]], want), b
        assert (keep[b, n[b]:] == -1).all() and np.array_equal(kept[b, :n[b]], w[b][want])


def test_a_long_sequence_alone(ic):
    say("evict one sequence of 300001")
    rng = np.random.default_rng(5)
    L, n_keep = 300001, 31007
    w = rng.lognormal(0, 2, (1, L)).astype(np.float32)
    w[0, rng.random(L) < 0.5] = 0.125                                            # the border among equal ones
    for nk in (n_keep, 200000):
        keep, n, kept = ic.evict_keep(torch.from_numpy(w).cuda(), nk, 4, 1000)
        order = np.lexsort((np.arange(4, L - 1000), -w[0, 4:L - 1000]))[:nk - 1004] + 4
        want = np.sort(np.concatenate([np.arange(4), order, np.arange(L - 1000, L)]))
        assert np.array_equal(keep.cpu().numpy()[0], want) and int(n[0]) == nk
        assert np.array_equal(kept.cpu().numpy()[0], w[0][want])


@pytest.mark.parametrize("sp, dp", [(0, 0), (64, 0), (0, 128), (64, 64)])
def test_rows_move_to_their_places(ic, sp, dp):
    say("compact, source page %d, destination page %d" % (sp, dp))
    rng = np.random.default_rng(sp + dp)
    lens, Lk, n_keep = [333, 150, 0, 200, 1], 333, 150
    B = len(lens)
    keep = np.full((B, n_keep), -1, dtype=np.int32)
    for b, n in enumerate(lens):
        m = min(n, n_keep)
        keep[b, :m] = np.sort(rng.choice(n, m, replace=False)) if m else keep[b, :m]
    keep[3, 5] = Lk                                                              # not a position: its row stays as it is
    s = Paged(ic, lens, Lk, sp, seed=1) if sp else None
    d = Paged(ic, [n_keep] * B, n_keep, dp, seed=2) if dp else None
    ns, nd = s.n_rows if sp else B * Lk, d.n_rows if dp else B * n_keep
    widths = [400, 256, 1152, 4, 12, 20]                                         # 4-bit rows, index keys, bf16 rows, scales; odd widths
    src = [torch.from_numpy(rng.integers(0, 1 << 32, (ns, w // 4), dtype=np.uint32).view(np.int32)).cuda() for w in widths]
    dst = [torch.full((nd, w // 4), 77, dtype=torch.int32, device="cuda") for w in widths]
    pairs = [(a if sp else a.view(B, Lk, -1), c if dp else c.view(B, n_keep, -1)) for a, c in zip(src, dst)]
    ic.cache_compact(pairs, torch.from_numpy(keep).cuda(), Lk, src_pc=s.pc if sp else None, dst_pc=d.pc if dp else None)
    torch.cuda.synchronize()
    for a, c in zip(src, dst):
        want = np.full(c.shape, 77, dtype=np.int32)
        an = a.cpu().numpy()
        for b in range(B):
            for j in range(n_keep):
                k = int(keep[b, j])
                if 0 <= k < Lk:
                    want[d.row(b, j) if dp else b * n_keep + j] = an[s.row(b, k) if sp else b * Lk + k]
        assert np.array_equal(c.cpu().numpy(), want)


def test_more_rows_than_the_caches_hold(ic):
    """Over 256 MB to write, in rows of 1152 and of 20 bytes."""
    say("compact 2 x 119001 rows of 1152 and 20 bytes")
    g = torch.Generator(device="cuda").manual_seed(3)
    B, Lk, n_keep = 2, 130000, 119001
    keep = torch.stack([torch.randperm(Lk, generator=g, device="cuda")[:n_keep].sort()[0] for _ in range(B)])
    keep[1, -3:] = -1
    src = [torch.randint(-(1 << 31), 1 << 31, (B, Lk, w // 4), generator=g, device="cuda").int() for w in (1152, 20)]
    dst = [torch.full((B, n_keep, w // 4), 77, dtype=torch.int32, device="cuda") for w in (1152, 20)]
    ic.cache_compact(list(zip(src, dst)), keep.int(), Lk)
    for a, c in zip(src, dst):
        assert torch.equal(c[0], a[0][keep[0]]) and torch.equal(c[1, :-3], a[1][keep[1, :-3]])
        assert bool((c[1, -3:] == 77).all())


def test_compaction_keeps_to_its_buffers(ic):
    """A page table that names pages the pools do not have."""
    table = torch.tensor([[1, 5, -3]], dtype=torch.int32, device="cuda")
    src, dst = torch.arange(128 * 4, dtype=torch.int32, device="cuda").view(128, 4), torch.zeros((1, 192, 4), dtype=torch.int32, device="cuda")
    keep = torch.arange(192, dtype=torch.int32, device="cuda")[None]
    ic.cache_compact([(src, dst)], keep, 192, src_pc=ic.paged_cache(None, table, 64))
    torch.cuda.synchronize()
    assert torch.equal(dst[0, :64], src[64:]) and not dst[0, 64:].any()


def test_together_as_a_server_uses_them(ic):
    """Decode steps over paged 4-bit caches with the indexer's selections: rows appended, attention, weights; then the caches are
    trimmed into fresh pages and attention over what stayed equals attention over the same rows of the old cache."""
    say("decode, evict, decode")
    B, Lk, page, k, n_keep = 3, 700, 64, 128, 320
    lens = [690, 400, 130]
    steps = 4
    pg = Paged(ic, [n + steps for n in lens], Lk, page, seed=3, ragged=False)
    g = torch.Generator().manual_seed(9)
    ik = torch.randn((pg.n_rows, 128), generator=g).to(torch.bfloat16).cuda()
    kv4 = torch.zeros((pg.n_rows, 400), dtype=torch.uint8, device="cuda")
    now = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pc = ic.paged_cache(now, pg.dev[1], page)
    ic.kv4_write(rows_of(1, B * 690, wide=False).reshape(B, 690, 576).cuda(), kv4, Lk=Lk, pc=pc)   # the prompts, ends aligned
    weight = torch.zeros((B, Lk), device="cuda")
    want_w = np.zeros((B, Lk))
    for t in range(steps):
        now += 1
        ic.kv4_write(torch.randn((B, 1, 576), generator=g).to(torch.bfloat16).cuda(), kv4, Lk=Lk, pc=pc)
        q = (torch.randn((B, 1, 32, 128), generator=g) / 11).to(torch.bfloat16).cuda()
        w = torch.rand((B, 1, 32), generator=g).cuda()
        Q = torch.randn((B, 1, 32, 576), generator=g).to(torch.bfloat16)
        idx = ic.indexer_topk_paged(q, ik, w, k, Lk, pc)
        O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, idx, SCALE, Lk=Lk, pc=pc, want_lse=True)
        probs = ic.attn_probs_kv4(Q.cuda(), kv4, idx, SCALE, lse, Lk=Lk, pc=pc)
        ic.attn_weight_add(probs, idx, weight)
        packed, ih = kv4.cpu().numpy(), idx.cpu().numpy()
        for b in range(B):
            valid = ih[b, 0] >= 0
            at = [pg.row(b, int(s)) if s >= 0 else 0 for s in ih[b, 0]]
            check_query(O[b, 0], lse[b, 0], probs[b, 0], kv4_ref.bf16_bits_to_f64(bits(Q))[b, 0], kv4_ref.unpack(packed[at]), valid)
            np.add.at(want_w[b], ih[b, 0][valid], probs[b, 0].cpu().double().numpy()[valid])
    assert np.all(np.abs(weight.cpu().double().numpy() - want_w) <= steps * 2.0 ** -24 * want_w + steps * 2.0 ** -48)
    keep, new_lens, kept = ic.evict_keep(weight, n_keep, n_first=4, n_recent=32, seq_lens=now)
    dst = Paged(ic, [n_keep] * B, n_keep, page, seed=4, ragged=False)
    kv4b, ikb = torch.zeros((dst.n_rows, 400), dtype=torch.uint8, device="cuda"), torch.zeros((dst.n_rows, 128), dtype=torch.bfloat16, device="cuda")
    new_pc = ic.paged_cache(new_lens, dst.dev[1], page)
    ic.cache_compact([(kv4, kv4b), (ik, ikb)], keep, Lk, src_pc=pc, dst_pc=new_pc)
    idx = ic.indexer_topk_paged(q, ikb, w, k, n_keep, new_pc)
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4b, idx, SCALE, Lk=n_keep, pc=new_pc, want_lse=True)
    old = torch.where(idx >= 0, keep.gather(1, idx[:, 0].clamp(min=0).long())[:, None], idx)       # the same rows where they were
    O2, lse2 = ic.sparse_attn_kv4(Q.cuda(), kv4, old.int().contiguous(), SCALE, Lk=Lk, pc=pc, want_lse=True)
    torch.cuda.synchronize()
    assert new_lens.cpu().tolist() == [n_keep, n_keep, 134]
    assert torch.equal(O, O2) and torch.equal(lse, lse2)                         # the same rows in the same order
    assert torch.equal(kept, torch.where(keep >= 0, weight.gather(1, keep.clamp(min=0).long()), torch.zeros_like(kept)))


def test_weights_of_the_most_positions(ic):
    """2^31 - 1 positions (8.6 GB), of which a few receive something."""
    say("weights of 2^31 - 1 positions")
    Lk = (1 << 31) - 1
    at = [0, 1, 4095, 4096, 16383, 16384, 1 << 30, Lk - 16384, Lk - 2, Lk - 1]
    idx = torch.tensor([[at + [-1, -(1 << 31)]]], dtype=torch.int32, device="cuda")
    p = torch.arange(1, len(at) + 3, device="cuda").float().reshape(1, 1, -1) / 64
    w = torch.zeros((1, Lk), device="cuda")
    ic.attn_weight_add(p, idx, w)
    got = w[0, torch.tensor(at, device="cuda")]
    assert torch.equal(got, p[0, 0, :len(at)])
    w[0, torch.tensor(at, device="cuda")] = 0
    assert not any(bool(c.any()) for c in w[0].split(1 << 28))


def test_more_rows_than_one_dimension_of_a_launch(ic):
    """2^29 + 5 rows of 4 bytes: more workgroups of 256 threads than 2^32 threads have."""
    n = (1 << 29) + 5
    say("compact %d rows" % n)
    src = torch.arange(n + 3, dtype=torch.int32, device="cuda").view(1, -1, 1)
    keep = torch.arange(3, n + 3, dtype=torch.int32, device="cuda").view(1, -1)
    keep[0, 7] = -1
    dst = torch.full((1, n, 1), -9, dtype=torch.int32, device="cuda")
    ic.cache_compact([(src, dst)], keep, n + 3)
    keep[0, 7] = -9
    assert torch.equal(dst.view(1, -1), keep)
