"""The layers' testing hooks on the host."""
from paper_2401_14110_b200 import binding as lba


def test_wait_override_numbers():
    lib = lba.load_library()
    assert lib.lba_set_wait_override(4) == -2 and lib.lba_set_wait_override(-1) == -2
    assert lib.lba_set_wait_override(1) == 0 and lib.lba_set_wait_override(0) == 0
