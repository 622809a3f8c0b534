"""A teacher's logits at the ends of their type, as masks leave them, with a temperature: a token's q depends on the logits' distances alone.  Against float64 on logits of the
same distances, by whose arithmetic (test_gpu_distil) the bounds are: a distance of 0 is exact, one past the type's range gives q = 0 on either side."""
import pytest
import torch

from test_gpu_distil import DT, check, inputs, reference, run

pytestmark = pytest.mark.gpu


# (entries looked at where they stand or sorted, tokens listed by every wave or by a launch)
@pytest.mark.parametrize("dtype,n,E,V,K", [("bf16", 20, 64, 300, 5), ("bf16", 20, 64, 300, 16), ("bf16", 300, 64, 511, 6), ("bf16", 300, 64, 511, 20), ("bf16", 1100, 64, 129, 9),
                                           ("f32", 20, 29, 301, 5), ("f32", 20, 29, 301, 30), ("f32", 300, 40, 900, 6), ("f32", 300, 40, 900, 16)])
@pytest.mark.parametrize("T", [0.5, 0.7, 2.0])
@pytest.mark.parametrize("teacher", ["f32", "bf16"])
def test_lowest_and_highest_logits(dtype, n, E, V, K, T, teacher):
    print(f"[distil] {dtype} {n}x{E} V={V} K={K} teacher {teacher} T {T}", flush=True)
    x, w, ids, t, d = inputs(n, E, V, K, dtype, n + V, teacher)
    ends, same = torch.finfo(DT[teacher]), t.clone()
    plain = t.isfinite()                             # (what is not there, or has q = 0, stays as it is)
    for rows, value in ((slice(0, None, 4), ends.min), (slice(2, None, 4), ends.max)):
        t[rows][plain[rows]], same[rows][plain[rows]] = value, 0.0
    masked = plain & (torch.arange(K, device="cuda") % 2 == 1)      # the first entry stays
    t[1::4][masked[1::4]], same[1::4][masked[1::4]] = ends.min, -float("inf")
    ref, tol, on = reference(x, w, ids, same, d, T, dtype)
    check(run(x, w, ids, t, d, T), ref, tol, f"{dtype} {n}x{E}x{V}, {K}, {teacher}, T {T}")
