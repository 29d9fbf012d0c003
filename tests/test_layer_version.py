"""The library's version tells a C program whether the operators around the recurrence are there (CPU only)."""
import paper_2605_11196_amd as vla


def test_the_entry_points_of_0_7_0_come_with_its_version():
    assert hasattr(vla.load_library(), "vla_delta_forward") and vla.version() >= 700
