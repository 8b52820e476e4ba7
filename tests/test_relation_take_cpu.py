"""BoxMemory.take is all or nothing, also where what fails is the tensor it returns (host code)."""
import pytest

from paper_1906_07155_amd import relation_head
from paper_1906_07155_amd.relation_head import BoxMemory


def test_slots_are_runs_of_places():
    m = BoxMemory(6, 2, 3, 1, 8, device="cpu")
    a = m.take([40, 1]).tolist()
    first, second = m.table[0]
    assert a == [first * 32 + t for t in range(32)] + [second * 32 + t for t in range(8)] + [m.table[1][0] * 32]
    b = m.take([64, 0]).tolist()                    # 24 places of the second page, a third one, then the first's again
    assert b[:24] == [second * 32 + t for t in range(8, 32)] and m.table[0][0] == second and m.used == [72, 1]
    assert b[24:56] == [m.table[0][1] * 32 + t for t in range(32)] and b[56:] == [m.table[0][2] * 32 + t for t in range(8)]


def test_a_tensor_that_cannot_be_made_takes_nothing(monkeypatch):
    m = BoxMemory(4, 1, 2, 1, 8, device="cpu")
    m.take([30])
    before = (list(m.free), [list(t) for t in m.table], list(m.used))

    def fail(*args, **kw):
        raise MemoryError("no room")
    with monkeypatch.context() as p:
        p.setattr(relation_head.torch, "tensor", fail)
        with pytest.raises(MemoryError):
            m.take([32])
    assert before == (m.free, m.table, m.used)
    with pytest.raises(ValueError, match="counts"):
        m.check([33])
    assert before == (m.free, m.table, m.used) and len(m.take([32])) == 32
