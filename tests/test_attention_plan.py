"""What the host decides for the policy's attention: launch grids, and which kernels a call's sizes lead to."""
from tests._plan import ask


def test_norm_and_rotation_of_any_number_of_tokens_is_one_launch():
    """HIP takes fewer than 2^32 threads in a dimension of a grid; every token has its wavefronts, and few others start."""
    sizes = [(1, 2), (8, 40), (5, 3), (16411, 40), ((1 << 24) + 1, 2), ((1 << 26) - 1, 2), (1 << 26, 2), ((1 << 26) + 5, 2),
             (2 ** 31 - 1024, 2), (2 ** 31 - 1024, 131072)]
    for (T, heads), a in zip(sizes, ask([f"rope {T} {heads}" for T, heads in sizes])):
        assert a["most"] < 2 ** 32 and a["units"] <= a["waves"] < a["units"] + 4 * (1 << 22), (T, heads, a)
