"""What the eviction entry points refuse about where their buffers lie and how long their sequences are, before anything is launched;
no GPU needed (addresses that nothing reads)."""
import pytest

FAR = 1 << 30


@pytest.fixture(scope="module")
def ic():
    import paper_2603_12201_amd as m
    m.lib()
    return m


def _evict(ic, B=2, Lk=1000, n_keep=400, weight=FAR, lens=2 * FAR, keep=3 * FAR, keep_lens=4 * FAR, kept=5 * FAR, have=1 << 40):
    return ic.lib().ic_evict_keep(B, Lk, weight, lens, n_keep, 4, 16, keep, keep_lens, kept, 6 * FAR, have, None)


def test_what_stays_is_not_written_over_what_is_read(ic):
    """Workgroups read lengths and weights while others write."""
    S = ic.Status
    for lens in (2 * FAR, None):                                                 # one sequence of a length in place, lengths in place
        assert _evict(ic, lens=lens, kept=FAR) == S.ERR_SHAPE                    # the weights in place
        assert _evict(ic, lens=lens, kept=FAR + 4 * (2 * 1000 - 1)) == S.ERR_SHAPE   # their last element
        assert _evict(ic, lens=lens, keep=FAR) == S.ERR_SHAPE
        assert _evict(ic, lens=lens, keep_lens=FAR + 4 * 1000) == S.ERR_SHAPE
        assert _evict(ic, lens=lens, keep=3 * FAR, kept=3 * FAR + 4 * (2 * 400 - 1)) == S.ERR_SHAPE
        assert _evict(ic, lens=lens, keep_lens=3 * FAR + 8) == S.ERR_SHAPE
        assert _evict(ic, lens=lens, keep_lens=5 * FAR) == S.ERR_SHAPE
    assert _evict(ic, keep_lens=2 * FAR) == S.ERR_SHAPE                          # the lengths in place
    assert _evict(ic, keep_lens=2 * FAR + 4) == S.ERR_SHAPE
    assert _evict(ic, keep=2 * FAR - 8 * 400 + 4) == S.ERR_SHAPE and _evict(ic, kept=2 * FAR) == S.ERR_SHAPE
    assert b"overlap" in ic.lib().ic_last_error()


def test_weights_are_not_written_over_what_is_read(ic):
    def add(probs=FAR, idx=2 * FAR, w_in=3 * FAR, w=4 * FAR):
        return ic.lib().ic_attn_weight_add(2, 3, 64, 1000, probs, idx, w_in, w, 6 * FAR, 1 << 40, None)

    S = ic.Status
    assert add(w=FAR) == S.ERR_SHAPE and add(w=FAR + 4 * (2 * 3 * 64 - 1)) == S.ERR_SHAPE and add(w=2 * FAR - 4 * (2 * 1000 - 1)) == S.ERR_SHAPE
    assert add(w=3 * FAR + 4) == S.ERR_SHAPE and add(w=3 * FAR - 4 * 1000) == S.ERR_SHAPE   # (the same address is in place, and allowed)


def test_sequences_whose_last_part_would_pass_32_bits(ic):
    """Parts of 8192 positions are numbered in 32 bits."""
    L, S = ic.lib(), ic.Status
    most = (1 << 31) - 8192
    assert L.ic_evict_keep_workspace(1, most) > 0 and _evict(ic, B=1, Lk=most, weight=1 << 40, have=0) == S.ERR_WORKSPACE
    for Lk in (most + 1, (1 << 31) - 1):
        assert L.ic_evict_keep_workspace(1, Lk) == 0
        assert _evict(ic, B=1, Lk=Lk, weight=1 << 40) == S.ERR_UNSUPPORTED


def test_chunks_of_the_most_query_rows(ic):
    """No chunk has more than 2^15 rows, whose sums fit 64 bits: 65536 chunks of 100 positions, 8 bytes each."""
    assert ic.lib().ic_attn_weight_add_workspace(1, (1 << 31) - 1, 1, 100) == 65536 * 100 * 8
    assert ic.lib().ic_attn_weight_add_workspace(1, 1 << 30, 1, 100) == 32768 * 100 * 8
