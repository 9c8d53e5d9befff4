"""A process may drive several GPUs from a thread each: host code keeps what it has found out per device, in no variable that the
devices' threads would share."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_09687_b200", "csrc")
LOCAL = re.compile(r"^\s+static\s+(?!const\b|constexpr\b|inline\b|cudaError_t\b.*\(|moin_status\b.*\()[\w:<>*& ]+\w\s*(=|;|\[|\{)")


def test_no_function_keeps_a_variable_of_its_own():
    found = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.cpp"))):
        with open(path) as f:
            found += [f"{os.path.basename(path)}:{i}: {line.strip()}" for i, line in enumerate(f, 1) if LOCAL.match(line) and "(" not in line.split("=")[0]]
    assert not found, found
