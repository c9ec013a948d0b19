"""The counters that the benchmark line quotes were taken with the sources as they are (no GPU)."""
import bench


def test_the_traffic_profile_belongs_to_the_current_sources():
    """A change of the dominant kernel's sources without new counters leaves the line's traffic null."""
    read = 180838400.0  # bytes of one launch's weights and activations, 7B gate/up at 8 rows
    traffic = bench.measured_traffic(read)
    assert traffic is not None, f"retake {bench.TRAFFIC_PROFILE}: its commands are in its head"
    assert read <= traffic <= 1.1 * read
