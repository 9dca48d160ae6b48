"""Host tests, which pass made-up addresses, are left out on a machine with a GPU, and no others are."""
import os
import re
import types

import pytest
import torch

import conftest


class Item:
    def __init__(self, address, gpu):
        self.module, self.gpu, self.marks = types.SimpleNamespace(**({} if address is None else {"P": address})), gpu, []

    def get_closest_marker(self, name):
        return object() if name == "gpu" and self.gpu else None

    def add_marker(self, mark):
        self.marks.append(mark.name)


@pytest.mark.parametrize("devices", [0, 1])
def test_which_are_left_out(monkeypatch, devices):
    monkeypatch.setattr(torch.cuda, "device_count", lambda: devices)
    items = [Item(conftest.MADE_UP, False), Item(conftest.MADE_UP, True), Item(None, False), Item(None, True), Item(5, False)]
    conftest.pytest_collection_modifyitems(items)
    assert [i.marks for i in items] == [["skip"] if devices else [], [], [], [], []]


def test_every_such_file_has_the_address():
    here = os.path.dirname(os.path.abspath(__file__))
    for name in sorted(os.listdir(here)):
        if name.startswith("test_") and name.endswith(".py"):
            for line in open(os.path.join(here, name)):
                m = re.match(r"(\w+) = (0x[0-9A-Fa-f]{9,})\b", line)
                assert not m or (m.group(1), int(m.group(2), 16)) == ("P", conftest.MADE_UP), (name, line)
