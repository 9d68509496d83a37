"""Host side of the torch interface of the layer operators, with a stand-in for the library: no GPU."""
import ctypes as C

from paper_2012_05396_b200 import layers as L


def test_the_marshalling_module_loads():
    assert L._marshal() is L._marshal() and callable(L._marshal().linear_forward)


class FakeLib:
    def __init__(self):
        self.destroyed = []

    def ssd_grad_list_destroy(self, handle):
        self.destroyed.append(handle.value)


def test_a_destroyed_list_has_no_address(monkeypatch):
    """Calls pass `address` on; after the list is gone there is none, which the entry points refuse, and it is not freed twice."""
    fake = FakeLib()
    monkeypatch.setattr(L, "lib", lambda: fake)
    lst = L.GradList.__new__(L.GradList)
    lst._h, lst.address = C.c_void_p(0x1230), 0x1230
    lst.ssd_grad_list_destroy()
    assert fake.destroyed == [0x1230] and lst.address == 0
    lst.ssd_grad_list_destroy()
    del lst
    assert fake.destroyed == [0x1230]


class FakeMarshal:
    def __init__(self):
        self.calls = []

    def clip(self, *args):
        self.calls.append(args)


def test_calls_name_the_table_and_its_stream(monkeypatch):
    """What ties the table's memory to the stream of a call (it may be another than the table's own) needs both."""
    fake = FakeMarshal()
    monkeypatch.setattr(L, "_torch", fake)
    monkeypatch.setattr(L, "lib", lambda: FakeLib())
    lst = L.GradList.__new__(L.GradList)
    lst._h, lst.address, lst.num_groups, lst.device = C.c_void_p(0), 0x1230, 3, type("D", (), {"index": 0})
    lst.table, lst.home = object(), 0x770
    L.ssd_clip_grad_norm(lst, 1.5)
    L.ssd_grad_norm(lst)
    assert fake.calls == [(0x1230, 0, 3, 1.5, 0, None, lst.table, 0x770), (0x1230, 0, 3, None, 0, None, lst.table, 0x770)]
