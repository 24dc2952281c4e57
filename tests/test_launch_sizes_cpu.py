"""The largest sizes that a call accepts can be launched: no launch has 2^32 threads in a
dimension, and together they have a workgroup for every row."""
import pytest

import launch_sizes

P = 1 << 40         # a pointer


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return launch_sizes.build(tmp_path_factory.mktemp("launch_sizes"))


@pytest.mark.parametrize("dtype", [0, 1])
def test_sample(fake, dtype):
    rows = [1, 70001, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, 1 << 24]
    got = launch_sizes.launches(fake, [
        ("d2moe_sample", [P, dtype, 3, B, 3, P, P, P, P, P, P, P, None]) for B in rows])
    for B, (status, log) in zip(rows, got):
        assert status == 0, B
        assert sum(n for _, n in log) == B and all("sample_kernel" in k for k, _ in log)
