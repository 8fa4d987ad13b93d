"""Tests that pass made-up device addresses to the library run only where no GPU is visible."""
import os
import pathlib
import re

import pytest
import torch

import conftest


class Item:
    def __init__(self, name, *keywords):
        self.path, self.keywords, self.marks = pathlib.Path(name), set(keywords), []

    def add_marker(self, mark):
        self.marks.append(mark.name)


@pytest.mark.parametrize("gpu", [False, True])
def test_where_tests_are_skipped(gpu, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_available", lambda: gpu)
    items = [Item("tests/test_operators_host.py"), Item("tests/test_host_api.py"), Item("tests/test_operators.py", "gpu"), Item("tests/test_asm_scan.py")]
    conftest.pytest_collection_modifyitems(None, items)
    assert [bool(i.marks) for i in items] == ([True, True, False, False] if gpu else [False, False, True, False])


def test_every_file_with_made_up_addresses_is_named():
    here = os.path.dirname(os.path.abspath(__file__))
    found = {n for n in os.listdir(here) if n.endswith(".py") and re.search(r"\b(FAKE|fake) = 0x", open(os.path.join(here, n)).read())}
    assert found == conftest.MADE_UP_ADDRESSES
