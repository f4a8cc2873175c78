"""One and two rows in the buffer: the kernel that gives every warp weight columns of its own, plain and gated."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_operators import BF, D, F32, FP, U, close, gated_reference, normal, offsets_of, wide

pytestmark = pytest.mark.gpu

# of one and two rows, with and without rows outside of the experts and experts without rows
LOADS = [([1], 0, 0), ([2], 0, 0), ([1, 1], 0, 0), ([0, 1, 0], 1, 0), ([0, 0, 1], 0, 1), ([1] + [0] * 40 + [1], 0, 0), ([0] * 35 + [2], 0, 0)]


def padded(t):
    """Rows a multiple of 8 apart, NaN between them, and the last row's end the buffer's end."""
    n = t.shape[-1]
    full = wide(t, -n % 8)
    flat = full.as_strided((full.numel() // n * (n + -n % 8) - (-n % 8),), (1,)).clone()
    return flat.as_strided(t.shape, full.stride())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("loads,before,behind", LOADS, ids=lambda x: "-".join(map(str, x[:3])) if isinstance(x, list) else str(x))
@pytest.mark.parametrize("N,K", [(40, 1001), (33, 13), (5, 7), (64, 64), (1, 1024 + 8), (130, 2056 + 3)])
def test_few_rows(loads, before, behind, N, K, dtype):
    off, o = offsets_of(loads, first=before)
    rows, E = o[-1] + behind, len(loads)
    x, w = padded(normal(rows, K, dtype=dtype)), padded(normal(E, N, K, seed=2, dtype=dtype, scale=0.25))
    if before:
        x[:before] = float("nan")
    start = normal(rows, N, seed=3, dtype=dtype)
    y, added = torch.full((rows, N), 7.0, dtype=dtype, device="cuda"), start.clone()
    hap.hap_expert_matmul(x, w, off, out=y)
    hap.hap_expert_matmul(x, w, off, out=added, accumulate=True)
    beside = wide(torch.zeros(rows, N, dtype=dtype, device="cuda"), 3)
    hap.hap_expert_matmul(x, w, off, out=beside)
    wide_out = torch.as_strided(beside, (rows, N + 3), (N + 3, 1))
    assert wide_out[:, N:].isnan().all()
    for t, untouched in ((y, torch.full_like(y, 7.0)), (added, start)):
        assert torch.equal(t[:before], untouched[:before]) and torch.equal(t[o[-1]:], untouched[o[-1]:])
    for e in range(E):
        i, j = o[e], o[e + 1]
        a, m = x[i:j].to(D), w[e].to(D)
        s = (K + 8) * U * (a.abs() @ m.abs().T)
        close(y[i:j], a @ m.T, s, dtype)
        close(added[i:j], a @ m.T + start[i:j].to(D), s + U * (a.abs() @ m.abs().T + start[i:j].to(D).abs()), dtype)
        assert torch.equal(beside[i:j], y[i:j])
    assert hap.hap_operator_status() == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("loads,before,behind", LOADS, ids=lambda x: "-".join(map(str, x[:3])) if isinstance(x, list) else str(x))
@pytest.mark.parametrize("F,H", [(40, 1001), (33, 13), (64, 64), (8, 2048), (131, 1032)])
def test_few_rows_gated(loads, before, behind, F, H, dtype):
    off, o = offsets_of(loads, first=before)
    rows, E = o[-1] + behind, len(loads)
    x, w = padded(normal(rows, H, dtype=dtype)), padded(normal(E, 2 * F, H, seed=1, dtype=dtype, scale=2.0 * H ** -0.5))
    gu, h = torch.full((rows, 2 * F), 7.0, dtype=dtype, device="cuda"), torch.full((rows, F), 7.0, dtype=dtype, device="cuda")
    hap.hap_expert_gated(x, w, off, gu=gu, h=h)
    only, none = hap.hap_expert_gated(x, w, off, keep=False)
    assert none is None and torch.equal(only[o[0]:o[-1]], h[o[0]:o[-1]])
    for t in (gu, h):
        assert (t[:before] == 7).all() and (t[o[-1]:] == 7).all()
    for e in range(E):
        i, j = o[e], o[e + 1]
        z, zoff, ref, hoff = gated_reference(x[i:j], w[e], F)
        close(gu[i:j], z, zoff, dtype)
        close(h[i:j], ref, hoff, dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("K", [1001, 13, 64, 5])
def test_one_row_whose_end_is_its_buffers(K, dtype):
    """Contiguous operands of a single row each: the row distance is nobody's."""
    off, _ = offsets_of([1])
    x, w = normal(1, K, dtype=dtype), normal(1, 1, K, seed=1, dtype=dtype)
    a, m = x.to(D), w[0].to(D)
    close(hap.hap_expert_matmul(x, w, off), a @ m.T, (K + 8) * U * (a.abs() @ m.abs().T), dtype)
    close(hap.hap_expert_matmul(x, w, off, out_dtype=F32), a @ m.T, (K + 8) * U * (a.abs() @ m.abs().T), F32)
