"""The sanitized check program calls every function that include/o5.h declares."""
import os
import re

from paper_1912_06680_amd import o5

HERE = os.path.dirname(os.path.abspath(__file__))


def test_every_entry_point_is_called():
    with open(os.path.join(HERE, "abi_host_check.cpp")) as f:
        text = f.read()
    missing = [name for name in o5.EXPORTED if not re.search(rf"\b{name}\s*\(", text)]
    assert not missing
