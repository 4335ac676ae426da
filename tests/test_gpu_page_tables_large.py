"""tasc_page_tables with as many slots as its limits allow."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_sequence_of_all_slots():
    """2^31 - 1 slots: of one sequence that is refused, and of one that is served and many rows behind it."""
    import torch
    import paper_2602_24174_amd as T
    cap, guard = 2 ** 31 - 1, 5
    one = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    slots = torch.full((cap + guard,), 9, dtype=torch.int32, device="cuda")
    for lens, rows, given in (((cap,), (cap,), 0), ((40, cap), (20, cap - 7), 20)):
        print(f"lengths {lens}, rows {rows}", flush=True)
        slots.fill_(9)
        table = torch.full((len(lens), 4), -1, dtype=torch.int32, device="cuda")
        row_off, summary = one(*[0] * (len(lens) + 1)), one(0, 0, 0)
        T.tasc_page_tables(one(*lens), one(*rows), None, one(5, 3, 8), table, row_off=row_off, slots=slots[:cap], summary=summary)
        assert (slots[cap:] == 9).all()
        assert slots[:given].tolist() == [([5, 3, 8][p // 16]) * 16 + p % 16 for p in range(40 - given, 40)][:given]
        assert int(slots[given:cap].max()) == -1 and int(slots[given:cap].min()) == -1
        assert summary.tolist() == [min(sum(rows), cap), 3 if given else 0, 1]
        assert row_off.tolist() == [0] + [min(sum(rows[:i + 1]), cap) for i in range(len(rows))]
