"""The DRAM traffic that the benchmark reports was captured from the kernel sources that are here."""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def test_traffic_of_the_default_kernel_is_known():
    import bench
    a = argparse.Namespace(ncu_traffic=None, config=3, kernel="mma", splits=0, contiguous=False)
    assert bench.ncu_traffic(a) == bench.NCU_CAPTURE["dram_bytes_per_launch"] > 1074266112   # the algorithm's bytes
