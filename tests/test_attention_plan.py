"""What the host decides for the policy's attention: launch grids, and which kernels a call's sizes lead to."""
from tests import test_gpu_attention_forms
from tests._plan import ask


def test_norm_and_rotation_of_any_number_of_tokens_is_one_launch():
    """HIP takes fewer than 2^32 threads in a dimension of a grid; every token has its wavefronts, and few others start."""
    sizes = [(1, 2), (8, 40), (5, 3), (16411, 40), ((1 << 24) + 1, 2), ((1 << 26) - 1, 2), (1 << 26, 2), ((1 << 26) + 5, 2),
             (2 ** 31 - 1024, 2), (2 ** 31 - 1024, 131072)]
    for (T, heads), a in zip(sizes, ask([f"rope {T} {heads}" for T, heads in sizes])):
        assert a["most"] < 2 ** 32 and a["units"] <= a["waves"] < a["units"] + 4 * (1 << 22), (T, heads, a)


def _forms(dtype, nq, nk, n, hq, hk, D, causal):
    return f"attention {nq} {nk} {n} {hq} {hk} {D} {1 if dtype == 'bf16' else 0} {1 if causal else 0}"


def _same(plan, want):
    got = {k: int(plan[k] > 1) if k.endswith("_parts") else plan[k] for k in want}
    return plan["ok"] == 1 and got == want


def test_gpu_cases_take_the_kernels_they_name():
    """A change of the cuts must not empty the GPU tests of the kernels they are there for."""
    cases = [(_forms(t, sum(q), sum(k), len(q), hq, hk, D, causal), want)
             for t, q, k, hq, hk, widths, causal, want in test_gpu_attention_forms.CASES for D in widths]
    cases += [(_forms(t, n, n, 1, hq, hk, D, True), want) for t, n, hq, hk, D, want in test_gpu_attention_forms.REACH]
    for (query, want), plan in zip(cases, ask([q for q, _ in cases])):
        assert _same(plan, want), (query, want, plan)


def test_the_gpu_cases_cover_the_forms():
    """Tiles of each size, whole walks and parts, at every compiled width, as far as any sizes lead to them."""
    cases = [(t, (D + 31) // 32, _forms(t, sum(q), sum(k), len(q), hq, hk, D, causal))
             for t, q, k, hq, hk, widths, causal, _ in test_gpu_attention_forms.CASES for D in widths]
    seen = set()
    for (t, width, _), plan in zip(cases, ask([c[2] for c in cases])):
        seen |= {(t, width, k, plan[k], int(plan[k + "_parts"] > 1)) for k in ("fwd", "dq", "dkdv")}
    tiles = {("bf16", "fwd"): [(32, 0), (32, 1), (64, 0), (128, 0), (128, 1)], ("bf16", "dq"): [(32, 0), (32, 1), (64, 0), (128, 0), (128, 1)],
             ("bf16", "dkdv"): [(32, 0), (32, 1), (64, 0), (64, 1), (128, 0)], ("f32", "fwd"): [(32, 0), (32, 1), (128, 0)],
             ("f32", "dq"): [(32, 0), (32, 1), (128, 0), (128, 1)], ("f32", "dkdv"): [(32, 0), (32, 1), (128, 0), (128, 1)]}
    missing = [(t, w, k, *form) for (t, k), forms in tiles.items() for form in forms for w in (1, 2, 3, 4) if (t, w, k, *form) not in seen]
    assert not missing, missing
