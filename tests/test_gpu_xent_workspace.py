"""The loss in a larger problem's workspace: bit for bit what it is in its own."""
import pytest
import torch

from paper_2502_02406_amd import binding as B

pytestmark = pytest.mark.gpu


# larger problems whose vocabulary is cut into pieces that are shorter than the smaller one's only piece; with more rows of the logits'
# gradient; without parts of dw where the smaller one has them
@pytest.mark.parametrize("dtype,small,large", [("bf16", (4096, 64, 131072), (4096, 64, 131073)), ("bf16", (2000, 64, 20000), (70000, 64, 20000)),
                                               ("bf16", (3000, 64, 700), (3000, 64, 20000)), ("f32", (4096, 8, 65536), (4096, 8, 65537))])
def test_results_are_the_same(dtype, small, large):
    print(f"[xent] {dtype} {small} in {large}", flush=True)
    n, E, V = small
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(n + V)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)
    x, w, d = rnd(n, E), rnd(V, E) * 0.2, torch.rand(n, generator=g, device="cuda")
    labels = torch.randint(-1, V, (n,), generator=g, device="cuda")
    results = []
    for size in (small, large):
        ws = torch.full((B.lvx_xent_workspace_bytes(*size, B.dtype_code(dt)),), 255, dtype=torch.uint8, device="cuda")
        loss, lse, dx, dw = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty_like(w)
        B.lvx_xent_fwd(x, w, labels, loss, lse, ws)
        ws.fill_(255)
        B.lvx_xent_bwd(x, w, labels, lse, d, dx, dw, ws)
        torch.cuda.synchronize()
        results.append((loss, lse, dx, dw))
    for a, b in zip(*results):
        assert a.isfinite().all() and torch.equal(a, b)
