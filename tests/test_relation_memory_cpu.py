"""The pages that BoxMemory hands out (host code; nothing here runs on a GPU)."""
import pytest

from paper_1906_07155_amd.relation_head import BoxMemory, RelationHead


def held(m, s):
    """Slots a stream remembers, from the table that the attention is given."""
    pages, lengths = m.pages_and_lengths()
    p = pages[s].tolist()
    return [p[t // 32] * 32 + t % 32 for t in range(int(lengths[s]))]


def test_slots_are_the_places_the_table_names():
    m = BoxMemory(8, 2, 4, 1, 8, device="cpu")
    first = m.take([40, 3]).tolist()
    assert len(set(first)) == 43 and held(m, 0) == first[:40] and held(m, 1) == first[40:]
    more = m.take([0, 30]).tolist()
    assert held(m, 1) == first[40:] + more and held(m, 0) == first[:40]
    assert m.table[1][0] != m.table[0][0] and len(m.free) == 8 - 2 - 2


def test_the_oldest_page_goes_first():
    m = BoxMemory(3, 1, 3, 1, 8, device="cpu")
    a = m.take([64]).tolist()
    b = m.take([20]).tolist()
    c = m.take([64]).tolist()           # 12 places are left, two pages more are needed
    assert len(set(c)) == 64 and held(m, 0) == (a + b + c)[64:]
    assert m.used == [84] and m.free == []


def test_no_slot_twice_in_one_call():
    m = BoxMemory(2, 1, 2, 1, 8, device="cpu")
    for c in (5, 32, 32, 31, 32, 1, 0, 32):
        s = m.take([c]).tolist()
        assert len(set(s)) == c and held(m, 0)[-c or 64:] == s


def test_a_pool_that_is_too_small_is_left_as_it_was():
    m = BoxMemory(3, 2, 3, 1, 8, device="cpu")
    m.take([33, 0])
    before = (list(m.free), [list(t) for t in m.table], list(m.used))
    with pytest.raises(RuntimeError, match="free pages"):
        m.take([32, 1])
    assert before == (m.free, m.table, m.used)
    m.forget(0)
    assert sorted(m.free) == [0, 1, 2] and held(m, 0) == []
    assert len(m.take([1, 33])) == 34


def test_refusals():
    with pytest.raises(ValueError, match="max_pages"):
        BoxMemory(4, 1, 1, 1, 8, device="cpu")
    with pytest.raises(ValueError, match="max_pages"):
        BoxMemory(4, 1, 5, 1, 8, device="cpu")
    m = BoxMemory(4, 2, 3, 1, 8, device="cpu")
    for counts in ([1], [1, -1], [65, 0]):
        with pytest.raises(ValueError, match="counts"):
            m.take(counts)
    for args in (dict(channels=60, heads=8), dict(channels=264, heads=2), dict(channels=64, heads=4, kv_heads=3)):
        with pytest.raises(ValueError):
            RelationHead(**args)
