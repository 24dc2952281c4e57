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


@pytest.mark.parametrize("x", [None, P])
@pytest.mark.parametrize("dtype", [0, 1])
def test_route_scored(fake, dtype, x):
    """Tokens by single waves, four a workgroup; their logits by tiles of 4 tokens, of one
    where a launch has no more than 4096 logits."""
    tokens, E = [5000, (1 << 26) - 4, (1 << 26) - 3, (1 << 26) + 5, (1 << 30) - 1, 1 << 30], 2
    got = launch_sizes.launches(fake, [
        ("d2moe_route_scored", [x, dtype, T, 8, P, P, E, 1, 1, P, 1, 1, 1, 1.0, P, P, 4, 2, 8,
                                [P] * 10, None]) for T in tokens])
    for T, (status, log) in zip(tokens, got):
        assert status == 0, T
        for kernel in ("scored_select_kernel", "gate_kernel"):
            groups = sum(n for k, n in log if kernel in k)
            if kernel[0] == "g":
                tail = T % (1 << 24)
                want = -(-T // 4) if tail * E > 4096 else (T - tail) // 4 + tail
                assert groups == (want if x else 0), T
            else:
                assert groups == -(-T // 4), T
