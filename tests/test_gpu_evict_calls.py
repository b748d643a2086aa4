"""Eviction and the 4-bit cache as servers may call them: captured and replayed, on a stream that is passed, within one pool."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4 import SCALE, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ic():
    import paper_2603_12201_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("B, Lk, n_keep", [(5, 900, 300), (2, 40000, 9000)])
def test_choice_and_move_captured(ic, B, Lk, n_keep):
    """Replayed on new weights and lengths, with eager calls between the replays."""
    print(f"[case] graph of choice and move, {B} x {Lk}", flush=True)
    w = torch.zeros((B, Lk), device="cuda")
    lens = torch.full((B,), Lk, dtype=torch.int32, device="cuda")
    src = torch.randint(0, 256, (B, Lk, 400), dtype=torch.uint8, device="cuda")
    dst = torch.zeros((B, n_keep, 400), dtype=torch.uint8, device="cuda")

    def step(to):
        keep, n, kept = ic.evict_keep(w, n_keep, 4, 32, seq_lens=lens)
        ic.cache_compact([(src, to)], keep, Lk)
        return keep, n, kept, to

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(dst)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(dst)
    for rep in range(4):
        g = torch.Generator().manual_seed(rep)
        w.copy_(torch.randint(0, 50, (B, Lk), generator=g).float())
        lens.copy_(torch.randint(1, Lk + 1, (B,), generator=g).int())
        lens[0] = Lk
        dst.fill_(rep)
        graph.replay()
        torch.cuda.synchronize()
        mine = [t.clone() for t in got]
        for a, b in zip(mine, step(torch.full_like(dst, rep))):
            assert torch.equal(a, b)


def test_rows_move_within_a_pool(ic):
    """One pool, the pages read and those written apart."""
    print("[case] one pool, two page tables", flush=True)
    B, Lk, n_keep, page = 3, 200, 70, 64
    order = np.random.default_rng(1).permutation(B * 4 + B * 2 + 3)
    st, dt = order[:B * 4].reshape(B, 4).astype(np.int32), order[B * 4:B * 6].reshape(B, 2).astype(np.int32)
    pools = [torch.randint(-(1 << 31), 1 << 31, (len(order) * page, w), dtype=torch.int64, device="cuda").int() for w in (100, 5)]
    keep = np.stack([np.sort(np.random.default_rng(b).permutation(Lk)[:n_keep]) for b in range(B)]).astype(np.int32)
    keep[2, 60:] = -1
    want = [p.cpu().numpy().copy() for p in pools]
    for a in want:
        was = a.copy()
        for b in range(B):
            for j, s in enumerate(keep[b]):
                if s >= 0:
                    a[dt[b, j // page] * page + j % page] = was[st[b, s // page] * page + s % page]
    ic.cache_compact([(p, p) for p in pools], torch.from_numpy(keep).cuda(), Lk, src_pc=ic.paged_cache(None, torch.from_numpy(st).cuda(), page),
                     dst_pc=ic.paged_cache(None, torch.from_numpy(dt).cuda(), page))
    for p, a in zip(pools, want):
        assert np.array_equal(p.cpu().numpy(), a)


def _calls(ic, stream):
    B, Lk, k = 3, 600, 500
    kv4 = torch.zeros((B, Lk, 400), dtype=torch.uint8, device="cuda")
    x = rows_of(3, B * Lk, wide=False).reshape(B, Lk, 576).cuda()
    Q = torch.randn((B, 1, 32, 576), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    idx = torch.arange(k, dtype=torch.int32, device="cuda").expand(B, 1, k).contiguous()
    w = torch.rand((B, Lk), generator=torch.Generator().manual_seed(2)).cuda()
    to = torch.zeros((B, 200, 400), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    s = dict(stream=stream)
    ic.kv4_write(x, kv4, **s)
    back = ic.kv4_read(kv4, B, Lk, **s)
    O, lse = ic.sparse_attn_kv4(Q, kv4, idx, SCALE, want_lse=True, **s)
    p = ic.attn_probs_kv4(Q, kv4, idx, SCALE, lse, **s)
    ic.attn_weight_add(p, idx, w, **s)
    keep, n, kept = ic.evict_keep(w, 200, 4, 16, **s)
    ic.cache_compact([(kv4, to)], keep, Lk, **s)
    torch.cuda.synchronize()
    return [kv4, back, O, lse, p, w, keep, n, kept, to]


def test_on_a_stream_that_is_passed(ic):
    print("[case] every call on a stream of its own", flush=True)
    want = _calls(ic, None)
    for _ in range(3):
        busy = torch.randn((4096, 4096), device="cuda")
        for _ in range(4):
            busy = busy @ busy
        for a, b in zip(want, _calls(ic, torch.cuda.Stream())):
            assert torch.equal(a, b)


def test_a_stream_of_another_device_is_refused(ic):
    class Elsewhere:
        device_index, cuda_stream = 1, 0

    kv4 = torch.zeros((2, 64, 400), dtype=torch.uint8, device="cuda")
    Q, idx = torch.zeros((2, 1, 32, 576), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 1, 16), dtype=torch.int32, device="cuda")
    w, keep = torch.zeros((2, 64), device="cuda"), torch.zeros((2, 8), dtype=torch.int32, device="cuda")
    s = dict(stream=Elsewhere())
    for f in (lambda: ic.kv4_write(Q[:, 0, :3].contiguous(), kv4, **s), lambda: ic.kv4_read(kv4, 2, 2, **s), lambda: ic.sparse_attn_kv4(Q, kv4, idx, SCALE, **s),
              lambda: ic.attn_probs_kv4(Q, kv4, idx, SCALE, torch.zeros((2, 1, 32), device="cuda"), **s),
              lambda: ic.attn_weight_add(torch.zeros((2, 1, 16), device="cuda"), idx, w, **s), lambda: ic.evict_keep(w, 8, **s),
              lambda: ic.cache_compact([(kv4, kv4[:, :8].contiguous())], keep, 64, **s)):
        with pytest.raises(ic.IcError, match="stream"):
            f()
