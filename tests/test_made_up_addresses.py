"""Calls with made-up addresses stay away from a GPU."""
import pathlib

import pytest

import conftest
import test_layer_operators_abi
import test_operators_abi

E_HIP = 7


class Item:
    def __init__(self, name, gpu):
        self.path, self.gpu, self.markers = pathlib.Path("tests") / name, gpu, []

    def get_closest_marker(self, name):
        return object() if self.gpu and name == "gpu" else None

    def add_marker(self, marker):
        self.markers.append(marker.name)


@pytest.mark.parametrize("gpus", [0, 1, 8])
def test_they_are_skipped_where_there_is_one(gpus):
    items = [Item("test_layer_operators_abi.py", False), Item("test_operators_abi.py", False), Item("test_abi.py", False),
             Item("test_layer_operators_abi.py", True), Item("test_rows_gpu.py", True), Item("test_oracle_pins.py", False)]
    conftest.skip_made_up_addresses(items, gpus)
    assert [i.markers for i in items] == [["skip"] if gpus else []] * 3 + [[]] * 3


def test_some_of_them_are_complete():
    """What the skip is for: without a GPU such a call passes every check and fails at the launch."""
    import torch
    if torch.cuda.device_count():
        pytest.skip("would be launched")
    assert test_layer_operators_abi.gates(dout=None)[0] == E_HIP and test_layer_operators_abi.rope(dq=None)[0] == E_HIP
    assert test_operators_abi.rows_calls(b=None)[0] == E_HIP
