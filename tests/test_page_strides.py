"""What the binding hands to the paged calls for tables of every layout: the distance of their rows as it is, so that the library can refuse rows that
overlap.  Nothing is launched: calls are recorded, and only those that the library refuses before it reads anything reach it."""
import pytest
import torch

from paper_2601_12247_amd import binding as B


class OnDevice(torch.Tensor):
    """A host tensor that says that it lies on device 0."""

    def get_device(self):
        return 0


def on(x):
    return x.as_subclass(OnDevice)


def i32(*shape):
    return on(torch.zeros(*shape, dtype=torch.int32))


def extend(table):
    n = table.shape[0]
    B.page_extend(i32(n), i32(n), table, i32(9), i32(1), 16, out=(i32(n), i32(1), i32(n + 1), i32(n), i32(n + 1), i32(7), i32(7)))


def trim(table):
    n = table.shape[0]
    B.page_trim(i32(n), i32(n), table, i32(9), i32(1), 16, out=(i32(n), i32(1), i32(n + 1)))


def attention(table):
    n = table.shape[0]
    q, kv = on(torch.zeros(n, 4, 64)), on(torch.zeros(4, 2, 16, 64))
    B.page_attention(q, kv, kv, table, i32(n), out=on(torch.zeros(n, 4, 64)), workspace=on(torch.zeros(16, dtype=torch.uint8)))


CALLS = [(extend, "pvf_page_extend", 6), (trim, "pvf_page_trim", 5), (attention, "pvf_page_attention", 11)]   # where the rows' distance is among the arguments; width is in front of it, the table in front of that
OVERLAP = [lambda: i32(5)[None].expand(3, 5), lambda: i32(9).as_strided((3, 5), (2, 1)), lambda: i32(7).as_strided((3, 5), (1, 1)), lambda: i32(1, 1).expand(4, 1),
           lambda: i32(2, 5)[:1].expand(3, 5)]
APART = [(lambda: i32(3, 5), 5), (lambda: i32(3, 9)[:, 2:7], 9), (lambda: i32(9, 5)[::3], 15), (lambda: i32(1, 5), 5), (lambda: i32(5)[None].expand(1, 5), 5),
         (lambda: i32(4, 1), 1), (lambda: i32(4, 6)[:, :1], 6)]


@pytest.fixture
def calls(monkeypatch):
    seen, place = [], {name: at for _, name, at in CALLS}

    def record(fn, dev, args):
        seen.append((fn.__name__, dev, args))
        width, apart = args[place[fn.__name__] - 1: place[fn.__name__] + 1]
        if apart < width:                                                       # what the library refuses
            B._check(fn(None, *args))

    monkeypatch.setattr(B, "_page_call", record)
    return seen


@pytest.mark.parametrize("call,name,at", CALLS)
@pytest.mark.parametrize("make", OVERLAP)
def test_tables_whose_rows_overlap_are_refused(calls, call, name, at, make):
    table = make()
    with pytest.raises(B.PvfError) as e:
        call(table)
    assert f"{name}: rows of the table are {table.stride(0)} apart and {table.shape[1]} wide" in str(e.value)
    assert calls[0][0] == name and calls[0][2][at] == table.stride(0)


@pytest.mark.parametrize("call,name,at", CALLS)
@pytest.mark.parametrize("make,apart", APART)
def test_rows_of_the_table_lie_where_the_tensor_says(calls, call, name, at, make, apart):
    table = make()
    call(table)
    (got, dev, args), = calls
    assert got == name and dev == 0 and args[at - 1] == table.shape[1] and args[at] == apart and args[at - 2] == table.data_ptr()


@pytest.mark.parametrize("call,name,at", CALLS)
def test_a_table_without_columns_is_no_overlap(calls, call, name, at):
    for table in (i32(3, 0), i32(3, 5)[:, :0]):
        calls.clear()
        call(table)
        assert calls[0][2][at - 1] == 0 and calls[0][2][at] >= 0
