"""The 4-bit cache on the GPU against 64 bits: rows written and read, attention over selected rows, their weights.

Tolerances.  Rows are exact.  Attention: P is rounded to bf16 (half a step, 2^-8 of the value, at most) and so is the output;
what a 32-bit sum of 576 products may be off in an exponent, zerr, moves P and the normaliser by that much each:
    |dO| <= (2^-8 + 2 zerr + 2^-20) sum p |v| + 2^-8 |O| + 2^-100,      |dlse| <= zerr + 2^-20 (1 + |lse|),
    |dprob| <= prob (2 zerr + 2^-20) + 2^-40
(2^-20: sums of 2048 terms and the exponential in 32 bits; 2^-100: P times a row's scale is dropped below the smallest normal
bf16, 2^-126, so each of 2^12 rows or fewer loses at most 6 2^-126, over a normaliser of at least 2^-12: 2^12 6 2^-126 2^12 < 2^-99.4,
and the rows of these tests are 2500 at most, 2^-100.1)."""
import math
import sys

import numpy as np
import pytest
import torch

from tests import kv4_ref

pytestmark = pytest.mark.gpu
SCALE = 1.0 / 24.0


def say(msg):
    print("[case] " + msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def ic():
    import paper_2603_12201_amd as m
    m.lib()
    return m


def bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def rows_of(seed, n, wide=True):
    """bf16 rows whose channels, blocks and rows differ in width."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, 576), generator=g)
    if wide:
        x = x * torch.exp(torch.randn((576,), generator=g)) * torch.exp2(torch.randint(-6, 7, (n, 4), generator=g).float()).repeat_interleave(144, 1)
    return x.to(torch.bfloat16)


class Paged:
    """Sequences of given lengths behind a page table whose pages are in an order of their own."""

    def __init__(self, ic, lens, Lk, page, seed=0, ragged=True):
        rng = np.random.default_rng(seed)
        self.lens, self.Lk, self.page = lens, Lk, page
        per = -(-Lk // page)
        used = [-(-n // page) for n in lens]
        order = rng.permutation(sum(used) + 2)                                   # two pages that belong to nobody
        table = np.full((len(lens), per), -1, dtype=np.int32)                    # entries behind a sequence are never read
        at = 0
        for b, u in enumerate(used):
            table[b, :u] = order[at:at + u]
            at += u
        self.table, self.n_rows = table, (sum(used) + 2) * page
        self.dev = (torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.from_numpy(table).cuda())
        self.pc = ic.paged_cache(self.dev[0] if ragged else None, self.dev[1], page)

    def row(self, b, s):
        return int(self.table[b, s // self.page]) * self.page + s % self.page


# ---- rows ----------------------------------------------------------------------------------------------------------

def test_rows_of_every_kind_are_packed_exactly(ic):
    say("4-bit rows: random bits, ties, zeros, denormals, infinities, NaN")
    rng = np.random.default_rng(1)
    x = bits(rows_of(3, 64))
    any_bits = rng.integers(0, 1 << 16, (200, 576)).astype(np.uint16)            # most of these blocks hold an infinity or a NaN
    fin = any_bits.copy()
    fin[(fin & 0x7F80) == 0x7F80] &= 0xBFFF
    small = (rng.integers(0, 1 << 7, (20, 576)) | (rng.integers(0, 2, (20, 576)) << 15)).astype(np.uint16)      # denormal
    steps = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6], dtype=np.float32)
    tie = np.zeros((8, 576), dtype=np.float32)
    for r in range(8):
        tie[r, :512] = rng.choice(steps, 512) * rng.choice([-1, 1], 512) * 2.0 ** (11 * r - 50)
        tie[r, 0::128] = 6 * 2.0 ** (11 * r - 50)
    edge = np.zeros((130, 576), dtype=np.uint16)                                 # a block's largest value: every step of one octave, at the ends of the range too
    for r in range(128):
        edge[r, 0::128] = [(127 << 7) + r, (127 << 7) + r | 0x8000, (228 << 7) + r, (28 << 7) + r, (1 << 7) + r]
    edge[128, :512] = 0x8000                                                     # minus zero
    edge[129, :512] = 0x7F7F                                                     # the largest finite
    rows = np.concatenate([x, any_bits, fin, small, (tie.view(np.uint32) >> 16).astype(np.uint16), edge])
    want = kv4_ref.pack(rows)
    t = torch.from_numpy(rows.view(np.int16).copy()).view(torch.bfloat16).cuda()[None]
    kv4 = torch.full((1, rows.shape[0], 400), 0xAB, dtype=torch.uint8, device="cuda")
    ic.kv4_write(t, kv4)
    back = ic.kv4_read(kv4, 1, rows.shape[0])
    torch.cuda.synchronize()
    got = kv4.cpu().numpy()[0]
    bad = np.argwhere(got != want)
    assert bad.size == 0, (bad[:5], got[tuple(bad[0])], want[tuple(bad[0])])
    u = kv4_ref.unpack(want)
    b = back.cpu()[0]
    assert np.array_equal(np.isnan(u[:, :512]), torch.isnan(b[:, :512]).numpy())
    assert np.array_equal(np.nan_to_num(u[:, :512]), np.nan_to_num(b[:, :512].double().numpy()))
    assert np.array_equal(bits(b)[:, 512:], rows[:, 512:])                       # the rotary part bit for bit


@pytest.mark.parametrize("B, Tn, Lk, pos0", [(1, 1, 1, 0), (3, 5, 40, 17), (2, 300, 257, -20), (1, 7, 64, 60), (2, 4, 10, 30)])
def test_rows_go_where_they_belong_and_nowhere_else(ic, B, Tn, Lk, pos0):
    say("write B=%d Tn=%d Lk=%d pos0=%d" % (B, Tn, Lk, pos0))
    x = rows_of(B + Tn, B * Tn).reshape(B, Tn, 576)
    want = np.full((B, Lk, 400), 0xAB, dtype=np.uint8)
    back = np.zeros((B, Tn, 576))
    p = kv4_ref.pack(bits(x))
    for b in range(B):
        for i in range(Tn):
            if 0 <= pos0 + i < Lk:
                want[b, pos0 + i] = p[b, i]
                back[b, i] = kv4_ref.unpack(p[b, i])
    kv4 = torch.full((B, Lk, 400), 0xAB, dtype=torch.uint8, device="cuda")
    ic.kv4_write(x.cuda(), kv4, pos0=pos0)
    out = ic.kv4_read(kv4, B, Tn, pos0=pos0)
    torch.cuda.synchronize()
    assert np.array_equal(kv4.cpu().numpy(), want)
    assert np.array_equal(out.cpu().double().numpy(), back)


@pytest.mark.parametrize("page", [0, 64, 256])
def test_ragged_rows_are_the_last_of_each_sequence(ic, page):
    lens, Lk, Tn = [300, 0, 2, 129, 64, 1], 300, 3
    say("ragged write, page %d" % page)
    B = len(lens)
    x = rows_of(page + 5, B * Tn).reshape(B, Tn, 576)
    p = kv4_ref.pack(bits(x))
    if page:
        pg = Paged(ic, lens, Lk, page)
        pc, n, row = pg.pc, pg.n_rows, pg.row
        kv4 = torch.full((n, 400), 0xAB, dtype=torch.uint8, device="cuda")
    else:
        ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
        pc, n, row = ic.paged_cache(ld), B * Lk, lambda b, s: b * Lk + s
        kv4 = torch.full((B, Lk, 400), 0xAB, dtype=torch.uint8, device="cuda")
    want, back = np.full((n, 400), 0xAB, dtype=np.uint8), np.zeros((B, Tn, 576))
    for b in range(B):
        for i in range(Tn):
            s = lens[b] - Tn + i
            if s >= 0:
                want[row(b, s)] = p[b, i]
                back[b, i] = kv4_ref.unpack(p[b, i])
    ic.kv4_write(x.cuda(), kv4, Lk=Lk, pc=pc)
    out = ic.kv4_read(kv4, B, Tn, Lk=Lk, pc=pc)
    torch.cuda.synchronize()
    assert np.array_equal(kv4.cpu().numpy().reshape(n, 400), want)
    assert np.array_equal(out.cpu().double().numpy(), back)


def test_pages_outside_the_pool_are_left_alone(ic):
    """Row numbers that no pool row has, from a table that holds them: host arithmetic first, then the kernels' own checks."""
    say("pages outside the pool")
    table = np.array([[0, -1, 2, 1 << 30, 3]], dtype=np.int32)                   # 64 rows a page, a pool of 3 pages
    there = [0 <= int(t) * 64 and int(t) * 64 + 63 < 3 * 64 for t in table[0]]
    assert there == [True, False, True, False, False]
    td = torch.from_numpy(table).cuda()
    pc = ic.paged_cache(None, td, 64)
    x = rows_of(9, 320).reshape(1, 320, 576)
    kv4 = torch.full((192, 400), 0xAB, dtype=torch.uint8, device="cuda")
    ic.kv4_write(x.cuda(), kv4, Lk=320, pc=pc)
    out = ic.kv4_read(kv4, 1, 320, Lk=320, pc=pc)
    torch.cuda.synchronize()
    p = kv4_ref.pack(bits(x))[0]
    got = kv4.cpu().numpy()
    assert np.array_equal(got[:64], p[:64]) and (got[64:128] == 0xAB).all() and np.array_equal(got[128:], p[128:192])
    assert not out[0, 64:128].any() and not out[0, 192:].any()
    # attention skips them
    Q = torch.randn((1, 1, 32, 576), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    idx = np.arange(320, dtype=np.int32)[None, None]
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, torch.from_numpy(idx).cuda(), SCALE, Lk=320, pc=pc, want_lse=True)
    probs = ic.attn_probs_kv4(Q.cuda(), kv4, torch.from_numpy(idx).cuda(), SCALE, lse, Lk=320, pc=pc)
    torch.cuda.synchronize()
    valid = np.zeros(320, dtype=bool)
    valid[:64] = valid[128:192] = True
    check_query(O[0, 0], lse[0, 0], probs[0, 0], kv4_ref.bf16_bits_to_f64(bits(Q))[0, 0], kv4_ref.unpack(p), valid)


# ---- attention -----------------------------------------------------------------------------------------------------

def check_query(O, lse, probs, Q, rows, valid):
    wo, wl, wp, zerr, pv = kv4_ref.attention(Q, rows, valid, SCALE)
    O, lse = O.cpu().double().numpy(), lse.cpu().double().numpy()
    tol = (2.0 ** -8 + 2 * zerr[:, None] + 2.0 ** -20) * pv + 2.0 ** -8 * np.abs(wo) + 2.0 ** -100
    err = np.abs(O - wo)
    assert np.all(err <= tol), (err.max(), (err / np.maximum(tol, 1e-300)).max())
    if not valid.any():
        assert np.all(np.isneginf(lse)) and not O.any()
    else:
        assert np.all(np.abs(lse - wl) <= zerr + 2.0 ** -20 * (1 + np.abs(wl)))
    if probs is not None:
        pr = probs.cpu().double().numpy()
        want = wp.mean(0)
        assert np.all(np.abs(pr - want) <= want * (2 * zerr.max() + 2.0 ** -20) + 2.0 ** -40)
        assert not pr[~valid].any()


def selection(rng, n, k, holes):
    """An index row over n visible positions: ascending distinct positions, then -1; or with holes and entries outside."""
    m = min(n, k)
    row = np.full(k, -1, dtype=np.int32)
    row[:m] = np.sort(rng.choice(n, m, replace=False)) if m else row[:m]
    if holes:
        row[rng.random(k) < 0.3] = -1
        if k > 3:
            row[rng.integers(0, k)] = 1 << 30
            row[rng.integers(0, k)] = -(1 << 31)
    return row


CASES = [
    # B, Tq, Lk, H, k, page (0: dense), ragged, holes
    (1, 1, 1, 32, 1, 0, False, False),            # one key
    (1, 1, 31, 1, 31, 0, False, False),           # one head, less than a tile
    (2, 1, 33, 32, 33, 0, False, False),          # a tile and a row
    (1, 1, 700, 32, 640, 64, True, False),        # split, paged
    (4, 1, 900, 17, 129, 128, True, True),
    (3, 2, 500, 20, 300, 0, True, True),
    (5, 1, 2500, 32, 2048, 64, True, False),      # the workload's k; short sequences
    (1, 300, 300, 32, 64, 0, False, False),       # a workgroup per query, no splits
    (2, 600, 640, 9, 100, 64, False, True),       # a wave per query, 1200 of them
    (1, 1030, 1030, 32, 257, 0, False, False),    # the same, causal rows, a last workgroup of two waves
    (1, 3, 400, 32, 2500, 0, False, False),       # more slots than keys
    (1, 256, 300, 31, 96, 128, True, False),      # a workgroup per query, three of its four waves with a tile
    (3, 171, 400, 32, 130, 64, True, True),       # 513 queries: the weights still four waves to a query, the attention one
]


@pytest.mark.parametrize("case", CASES)
def test_attention_and_weights_match_64_bits(ic, case):
    B, Tq, Lk, H, k, page, ragged, holes = case
    say("4-bit attention B=%d Tq=%d Lk=%d H=%d k=%d page=%d ragged=%s holes=%s" % case)
    rng = np.random.default_rng(Tq + Lk)
    lens = [Lk] * B
    if ragged:
        lens = [Lk] + [int(rng.integers(0, Lk)) for _ in range(B - 1)]
        if B > 1:
            lens[-1] = 1 if B % 2 else 0
    pg = Paged(ic, lens, Lk, page, seed=B, ragged=ragged) if page else None
    n = pg.n_rows if page else B * Lk
    x = rows_of(Lk, n, wide=False)
    packed = kv4_ref.pack(bits(x))
    dead = np.ones(n, dtype=bool)                                                # rows of no sequence hold what they like: here NaN
    for b in range(B):
        for s in range(lens[b]):
            dead[pg.row(b, s) if page else b * Lk + s] = False
    packed[dead] = 0xFF
    row = pg.row if page else (lambda b, s: b * Lk + s)
    kv4 = torch.from_numpy(packed).cuda()
    kv4 = kv4 if page else kv4.view(B, Lk, 400)
    Q = (1.5 * torch.randn((B, Tq, H, 576), generator=torch.Generator().manual_seed(k))).to(torch.bfloat16)
    idx = np.stack([np.stack([selection(rng, max(0, lens[b] - Tq + 1 + t), k, holes) for t in range(Tq)]) for b in range(B)])
    idx[0, -1, 0] = -1
    if Tq > 1:
        idx[0, 0] = -1                                                           # a row that selects nothing
    if ragged and k > 2 and lens[-1] < Lk:
        idx[-1, 0, k // 2] = lens[-1]                                            # a position behind the sequence
    pc = pg.pc if page else ic.paged_cache(torch.tensor(lens, dtype=torch.int32, device="cuda")) if ragged else None
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, torch.from_numpy(idx).cuda(), SCALE, Lk=Lk, pc=pc, want_lse=True)
    probs = ic.attn_probs_kv4(Q.cuda(), kv4, torch.from_numpy(idx).cuda(), SCALE, lse, Lk=Lk, pc=pc)
    again = ic.sparse_attn_kv4(Q.cuda(), kv4, torch.from_numpy(idx).cuda(), SCALE, Lk=Lk, pc=pc)
    torch.cuda.synchronize()
    assert torch.equal(again, O)
    Qf = kv4_ref.bf16_bits_to_f64(bits(Q))
    some = range(Tq) if Tq <= 3 else sorted(set([0, 1, Tq // 2, Tq - 2, Tq - 1]) | set(rng.integers(0, Tq, 12).tolist()))
    for b in range(B):
        for t in some:
            valid = (idx[b, t] >= 0) & (idx[b, t] < lens[b])
            at = [row(b, int(s)) if v else 0 for s, v in zip(idx[b, t], valid)]
            check_query(O[b, t], lse[b, t], probs[b, t], Qf[b, t], np.nan_to_num(kv4_ref.unpack(packed[at])), valid)


def test_large_logits_and_rising_maxima(ic):
    """Rows in an order of rising scores, hundreds of units apart, so that the reference of a row has to follow; and a row of one
    huge score."""
    say("rising maxima")
    k = Lk = 512
    x = rows_of(11, Lk, wide=False)
    Q = torch.randn((1, 2, 32, 576), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    x[:, 512:] = 0
    Q[0, :, :, 512:] = 0
    Q[0, 0, :, 512] = 24.0
    x[:, 512] = (torch.arange(Lk).float() * 0.75).to(torch.bfloat16)             # z rises by 0.75 a row, 384 in all
    Q[0, 1, :, 513] = 24.0
    x[100, 513] = 3000.0
    kv4 = torch.empty((1, Lk, 400), dtype=torch.uint8, device="cuda")
    ic.kv4_write(x.cuda()[None], kv4)
    for order in (np.arange(k), np.arange(k)[::-1].copy()):
        idx = np.broadcast_to(order.astype(np.int32), (1, 2, k)).copy()
        O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, torch.from_numpy(idx).cuda(), SCALE, want_lse=True)
        big = torch.from_numpy(np.broadcast_to(idx, (1, 2, k))).expand(700, 2, k).contiguous()       # the same a wave each
        O2, lse2 = ic.sparse_attn_kv4(Q.cuda().expand(700, 2, 32, 576).contiguous(), kv4.expand(700, Lk, 400).contiguous(), big.cuda(), SCALE, want_lse=True)
        torch.cuda.synchronize()
        u = kv4_ref.unpack(kv4.cpu().numpy()[0])[order]
        Qf = kv4_ref.bf16_bits_to_f64(bits(Q))
        for t in range(2):
            check_query(O[0, t], lse[0, t], None, Qf[0, t], u, np.ones(k, dtype=bool))
            check_query(O2[699, t], lse2[699, t], None, Qf[0, t], u, np.ones(k, dtype=bool))


def test_numbers_that_are_none_stay_with_their_rows(ic):
    """A selected block that is not a number makes its query NaN, and no other."""
    say("NaN in a selected row")
    x = rows_of(12, 400, wide=False)
    x[7, 3] = float("nan")
    Q = torch.randn((1, 2, 32, 576), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    kv4 = torch.empty((1, 400, 400), dtype=torch.uint8, device="cuda")
    ic.kv4_write(x.cuda()[None], kv4)
    idx = np.stack([np.arange(0, 100), np.arange(100, 200)])[None].astype(np.int32)
    for rep in (1, 600):
        O, lse = ic.sparse_attn_kv4(Q.cuda().expand(rep, 2, 32, 576).contiguous(), kv4.expand(rep, 400, 400).contiguous(),
                                    torch.from_numpy(idx).cuda().expand(rep, 2, 100).contiguous(), SCALE, want_lse=True)
        assert torch.isnan(O[:, 0]).all() and torch.isnan(lse[:, 0]).all()
        assert torch.isfinite(O[:, 1].float()).all() and torch.isfinite(lse[:, 1]).all()


@pytest.mark.parametrize("nq", [2, 600])
def test_a_position_named_more_than_once_counts_as_often(ic, nq):
    say(f"entries that repeat, {nq} queries")
    rng = np.random.default_rng(nq)
    Lk, k = 50, 200
    x = rows_of(6, Lk, wide=False)
    packed = kv4_ref.pack(bits(x))
    Q = torch.randn((1, nq, 32, 576), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    idx = rng.integers(0, Lk, (1, nq, k)).astype(np.int32)
    idx[0, 0] = 7
    kv4, at = torch.from_numpy(packed).cuda().view(1, Lk, 400), torch.from_numpy(idx).cuda()
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, at, SCALE, want_lse=True)
    probs = ic.attn_probs_kv4(Q.cuda(), kv4, at, SCALE, lse)
    weight = ic.attn_weight_add(probs, at, torch.zeros((1, Lk), device="cuda"))
    rows = kv4_ref.unpack(packed)
    for t in (0, 1, nq - 1):
        check_query(O[0, t], lse[0, t], probs[0, t], kv4_ref.bf16_bits_to_f64(bits(Q))[0, t], rows[idx[0, t]], np.ones(k, dtype=bool))
    want = np.zeros(Lk)
    np.add.at(want, idx.ravel(), probs.double().cpu().numpy().ravel())
    # each entry down to 2^-48, the sum rounded to fp32
    assert np.all(np.abs(weight[0].double().cpu().numpy() - want) <= nq * k * 2.0 ** -48 + want * 2.0 ** -24)


def test_calls_at_once_on_two_streams(ic):
    """The same operators on two streams with nothing between them: what each leaves is what it leaves alone."""
    say("two streams at once")
    jobs = []
    for i, (B, k) in enumerate([(3, 700), (5, 300)]):
        Lk = 900
        kv4 = torch.from_numpy(kv4_ref.pack(bits(rows_of(40 + i, B * Lk, wide=False)))).cuda().view(B, Lk, 400)
        Q = torch.randn((B, 1, 32, 576), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda()
        idx = torch.stack([torch.randperm(Lk, generator=torch.Generator().manual_seed(9 * i + b))[:k].sort()[0].int() for b in range(B)])[:, None].contiguous().cuda()
        jobs.append((Q, kv4, idx))

    def run(Q, kv4, idx):
        O, lse = ic.sparse_attn_kv4(Q, kv4, idx, SCALE, want_lse=True)
        p = ic.attn_probs_kv4(Q, kv4, idx, SCALE, lse)
        w = ic.attn_weight_add(p, idx, torch.zeros((Q.shape[0], kv4.shape[1]), device="cuda"))
        return [O, lse, p, w] + list(ic.evict_keep(w, 400, 4, 50))

    alone = [run(*j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(4):
        got = []
        for st, j in zip(streams, jobs):
            with torch.cuda.stream(st):
                got.append([run(*j) for _ in range(3)])
        torch.cuda.synchronize()
        for want, runs in zip(alone, got):
            for r in runs:
                assert all(torch.equal(a, b) for a, b in zip(want, r))


@pytest.mark.parametrize("nq", [1, 700])
def test_a_block_without_numbers_is_none_whatever_its_codes(ic, nq):
    """The exponent byte 255 beside any codes, and queries of either sign: an infinity of one sign would leave the softmax."""
    say(f"exponent byte 255, {nq} queries")
    idx = torch.arange(64, dtype=torch.int32, device="cuda").expand(1, nq, 64).contiguous()
    for code, block, sign in [(0x00, 0, 1.0), (0x11, 1, -1.0), (0x11, 2, 1.0), (0x99, 3, 1.0), (0x77, 0, -1.0), (0xFF, 2, 1.0)]:
        kv4 = torch.zeros((1, 64, 400), dtype=torch.uint8, device="cuda")
        kv4[..., :256] = 0x11
        kv4[..., 384:388] = 127
        kv4[0, 5, 64 * block:64 * block + 64] = code
        kv4[0, 5, 384 + block] = 255
        Q = torch.full((1, nq, 32, 576), sign, dtype=torch.bfloat16, device="cuda")
        O, lse = ic.sparse_attn_kv4(Q, kv4, idx, SCALE, want_lse=True)
        probs = ic.attn_probs_kv4(Q, kv4, idx, SCALE, lse)
        assert O.isnan().all() and lse.isnan().all() and probs.isnan().all(), (hex(code), block, sign)
        back = ic.kv4_read(kv4, 1, 64)
        assert back[0, 5, 128 * block:128 * block + 128].isnan().all() and int(back.isnan().sum()) == 128


def test_wide_scales(ic):
    """Blocks whose widths are 2^-60 and 2^60: the scales go into P's exponent."""
    say("wide scales")
    x = rows_of(13, 96, wide=False).float()
    x[:, 0:128] *= 2.0 ** -60
    x[:, 128:256] *= 2.0 ** 60
    x[::2, 256:384] = 0
    x = x.to(torch.bfloat16)
    Q = torch.randn((1, 1, 32, 576), generator=torch.Generator().manual_seed(8))
    Q[..., 128:256] = 0
    Q = Q.to(torch.bfloat16)
    kv4 = torch.empty((1, 96, 400), dtype=torch.uint8, device="cuda")
    ic.kv4_write(x.cuda()[None], kv4)
    idx = torch.arange(96, dtype=torch.int32).reshape(1, 1, 96)
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, idx.cuda(), SCALE, want_lse=True)
    torch.cuda.synchronize()
    check_query(O[0, 0], lse[0, 0], None, kv4_ref.bf16_bits_to_f64(bits(Q))[0, 0], kv4_ref.unpack(kv4.cpu().numpy()[0]), np.ones(96, dtype=bool))


@pytest.mark.parametrize("nq", [1, 300, 700])
def test_many_slots_of_the_largest_values(ic, nq):
    """16384 rows of 6 2^100, all but the first 128 of them 11.5 powers of two heavier: the sums must stay finite."""
    say(f"16384 slots, {nq} queries")
    k = 16384
    packed = np.zeros((1, k, 400), dtype=np.uint8)
    packed[..., :256] = 0x77
    packed[..., 384:388] = 227
    rope = torch.zeros((k, 64), dtype=torch.bfloat16)
    rope[128:, 0] = 11.5 / (1.4427 * SCALE)
    packed[0, :, 256:384] = rope.view(torch.uint8).numpy()
    Q = torch.zeros((1, nq, 32, 576), dtype=torch.bfloat16)
    Q[..., 512] = 1.0
    idx = torch.arange(k, dtype=torch.int32, device="cuda").expand(1, nq, k).contiguous()
    O, lse = ic.sparse_attn_kv4(Q.cuda(), torch.from_numpy(packed).cuda(), idx, SCALE, want_lse=True)
    # every row holds the same value, and so does their mean, but for roundings: 2^-8 of each P, 2^-8 of O, and in the two
    # sums, whose longest chains have 16384 / 2 and 16384 terms, at most 2^-11 and 2^-10
    x = O.double().cpu().numpy() / (6.0 * 2.0 ** 100)
    assert np.all(np.abs(x - 1.0) <= 2.0 ** -7 + 2.0 ** -9), (x.min(), x.max())
    s = SCALE * rope[:, 0].double().numpy()
    want = np.log(np.exp(s - s.max()).sum()) + s.max()
    assert np.all(np.abs(lse.double().cpu().numpy() - want) <= 2.0 ** -11 + 2.0 ** -20 * (1 + want))


def test_rows_behind_4_gib(ic):
    """A pool of 11.2 million rows (4.5 GB): row offsets pass 32 bits."""
    n = 175000 * 64
    say("a pool of %d rows" % n)
    kv4 = torch.empty((n, 400), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[174999, 3, 170000]], dtype=torch.int32, device="cuda")
    pc = ic.paged_cache(None, table, 64)
    x = rows_of(14, 192, wide=False)
    ic.kv4_write(x.cuda()[None], kv4, Lk=192, pc=pc)
    want = kv4_ref.pack(bits(x))
    for p, page in enumerate((174999, 3, 170000)):
        assert np.array_equal(kv4[page * 64:page * 64 + 64].cpu().numpy(), want[64 * p:64 * p + 64])
    Q = torch.randn((1, 1, 32, 576), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    idx = torch.arange(192, dtype=torch.int32).reshape(1, 1, 192)
    O, lse = ic.sparse_attn_kv4(Q.cuda(), kv4, idx.cuda(), SCALE, Lk=192, pc=pc, want_lse=True)
    probs = ic.attn_probs_kv4(Q.cuda(), kv4, idx.cuda(), SCALE, lse, Lk=192, pc=pc)
    torch.cuda.synchronize()
    check_query(O[0, 0], lse[0, 0], probs[0, 0], kv4_ref.bf16_bits_to_f64(bits(Q))[0, 0], kv4_ref.unpack(want), np.ones(192, dtype=bool))


def test_binding_refuses_mismatched_tensors(ic):
    kv4 = torch.zeros((2, 64, 400), dtype=torch.uint8, device="cuda")
    x = torch.zeros((2, 3, 576), dtype=torch.bfloat16, device="cuda")
    Q = torch.zeros((2, 1, 32, 576), dtype=torch.bfloat16, device="cuda")
    idx = torch.zeros((2, 1, 16), dtype=torch.int32, device="cuda")
    lens = torch.full((3,), 64, dtype=torch.int32, device="cuda")
    table = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    bad = [
        lambda: ic.kv4_write(x[:1], kv4), lambda: ic.kv4_write(x[..., :512].contiguous(), kv4), lambda: ic.kv4_write(x.float(), kv4),
        lambda: ic.kv4_write(x, kv4[..., :384].contiguous()), lambda: ic.kv4_write(x, kv4.view(128, 400)), lambda: ic.kv4_write(x, kv4, Lk=65),
        lambda: ic.kv4_write(x, kv4, pc=ic.paged_cache(lens)), lambda: ic.kv4_write(x, kv4.view(128, 400), pc=ic.paged_cache(None, table, 64)),
        lambda: ic.kv4_write(x.transpose(0, 1), kv4), lambda: ic.kv4_read(kv4, 3, 2), lambda: ic.kv4_read(kv4, 2, 2, out=x),
        lambda: ic.sparse_attn_kv4(Q[:1], kv4, idx, SCALE), lambda: ic.sparse_attn_kv4(Q, kv4, idx.long(), SCALE),
        lambda: ic.sparse_attn_kv4(Q, kv4, idx, SCALE, out=Q), lambda: ic.sparse_attn_kv4(Q[..., :64].contiguous(), kv4, idx, SCALE),
        lambda: ic.attn_probs_kv4(Q, kv4, idx, SCALE, torch.zeros((2, 1, 31), device="cuda")),
        lambda: ic.sparse_attn_kv4(Q.view(-1)[4:4 + 576 * 32].view(1, 1, 32, 576), kv4[:1], idx[:1], SCALE),      # 8 bytes off
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ic.IcError):
            f()
            pytest.fail("call %d went through" % i)


def test_tensors_away_from_the_current_device_are_refused(ic, monkeypatch):
    from paper_2603_12201_amd import binding
    kv4 = torch.zeros((2, 64, 400), dtype=torch.uint8, device="cuda")
    x = torch.zeros((2, 3, 576), dtype=torch.bfloat16, device="cuda")
    Q = torch.zeros((2, 1, 32, 576), dtype=torch.bfloat16, device="cuda")
    idx = torch.zeros((2, 1, 16), dtype=torch.int32, device="cuda")
    lse, weight, keep = torch.zeros((2, 1, 32), device="cuda"), torch.zeros((2, 64), device="cuda"), torch.zeros((2, 8), dtype=torch.int32, device="cuda")
    calls = [
        lambda: ic.kv4_write(x, kv4), lambda: ic.kv4_read(kv4, 2, 2), lambda: ic.sparse_attn_kv4(Q, kv4, idx, SCALE),
        lambda: ic.attn_probs_kv4(Q, kv4, idx, SCALE, lse), lambda: ic.attn_weight_add(torch.zeros((2, 1, 16), device="cuda"), idx, weight),
        lambda: ic.evict_keep(weight, 8), lambda: ic.cache_compact([(kv4, kv4[:, :8].contiguous())], keep, 64),
    ]
    for f in calls:
        f()
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    for f in calls:
        with pytest.raises(ic.IcError):
            f()


def test_captured_and_on_another_stream(ic):
    """Write, attention and weights captured once and replayed on new contents, beside eager work."""
    say("graph of write, attention, weights")
    B, Lk, k = 6, 500, 256
    x = torch.empty((B, 1, 576), dtype=torch.bfloat16, device="cuda")
    base = rows_of(21, B * Lk, wide=False).reshape(B, Lk, 576).cuda()
    kv4 = torch.empty((B, Lk, 400), dtype=torch.uint8, device="cuda")
    ic.kv4_write(base, kv4)
    lens = torch.full((B,), 400, dtype=torch.int32, device="cuda")
    pc = ic.paged_cache(lens)
    Q = torch.empty((B, 1, 32, 576), dtype=torch.bfloat16, device="cuda")
    idx = torch.arange(399 - k + 1, 400, dtype=torch.int32, device="cuda").expand(B, 1, k).contiguous()

    def step(w):
        ic.kv4_write(x, kv4, Lk=Lk, pc=pc)
        O, lse = ic.sparse_attn_kv4(Q, kv4, idx, SCALE, Lk=Lk, pc=pc, want_lse=True)
        p = ic.attn_probs_kv4(Q, kv4, idx, SCALE, lse, Lk=Lk, pc=pc)
        return O, lse, p, ic.attn_weight_add(p, idx, w, out=torch.empty_like(w))

    weight = torch.rand((B, Lk), generator=torch.Generator().manual_seed(0)).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(weight)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(weight)
    for rep in range(4):
        g = torch.Generator().manual_seed(rep)
        x.copy_(torch.randn(x.shape, generator=g).to(torch.bfloat16))
        Q.copy_(torch.randn(Q.shape, generator=g).to(torch.bfloat16))
        lens.fill_(400 - rep)
        graph.replay()
        torch.cuda.synchronize()
        mine = [t.clone() for t in got]
        want = step(weight)
        torch.cuda.synchronize()
        for a, b in zip(mine, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("page", [0, 64])
def test_lengths_beyond_the_bound_leave_out_the_rows_behind_it(ic, page):
    """Row i goes to seq_lens[b] - Tn + i, also where that is behind Lk: such rows are left out, the others keep their positions."""
    B, Lk, Tn = 4, 100, 6
    lens = [100, 103, 106, 1 << 30]
    say("write behind the bound, page %d" % page)
    x = rows_of(31, B * Tn).reshape(B, Tn, 576)
    p = kv4_ref.pack(bits(x))
    pg = Paged(ic, [Lk] * B, Lk, page) if page else None
    n = pg.n_rows if page else B * Lk
    pc = ic.paged_cache(torch.tensor(lens, dtype=torch.int32, device="cuda"), pg.dev[1] if page else None, page)
    kv4 = torch.full((n, 400) if page else (B, Lk, 400), 0xAB, dtype=torch.uint8, device="cuda")
    want, back = np.full((n, 400), 0xAB, dtype=np.uint8), np.zeros((B, Tn, 576))
    for b in range(B):
        for i in range(Tn):
            s = lens[b] - Tn + i
            if s < Lk:
                want[pg.row(b, s) if page else b * Lk + s] = p[b, i]
                back[b, i] = kv4_ref.unpack(p[b, i])
    ic.kv4_write(x.cuda(), kv4, Lk=Lk, pc=pc)
    out = ic.kv4_read(kv4, B, Tn, Lk=Lk, pc=pc)
    torch.cuda.synchronize()
    assert np.array_equal(kv4.cpu().numpy().reshape(n, 400), want)
    assert np.array_equal(out.cpu().double().numpy(), back)
