"""Outputs in the place of inputs: rows the same distance apart, or the call is refused (which is checked without a GPU)."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from paper_2609_39350_b200.tokens import _lib

INVALID = 1
A, B = 1 << 20, 1 << 21         # aligned addresses that are never read


def test_other_distances_are_refused():
    L = _lib()

    def norm(y=A, ldy=72, x=A, ldx=64):
        return L.hap_layer_norm(0, 0, 1, 100, 64, x, ldx, None, None, 1e-5, y, ldy, None, None, None)

    def norm_backward(dx=A, lddx=72, **at):
        p = dict(dy=B, x=B, b=B) | at
        return L.hap_layer_norm_backward(0, 0, 0, 0, 1, 100, 64, p["dy"], 64, p["x"], 64, None, B, B, p["b"], 64, dx, lddx, None, None, None, 0, None)

    def combine(out=A, ldo=72, base=A, ldb=64):
        return L.hap_expert_combine(0, 100, 2, 64, 16, B, 64, B, None, base, ldb, out, ldo, None)

    assert norm() == INVALID and norm(ldy=64, ldx=72) == INVALID
    assert norm_backward(dy=A) == INVALID and norm_backward(x=A) == INVALID and norm_backward(b=A) == INVALID
    assert combine() == INVALID and combine(ldo=64, ldb=72) == INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("rows,H", [(1, 8), (7, 264), (5, 1001), (300, 8200), (2000, 72), (2500, 520), (1500, 1001), (3, 16384)])
def test_norms_in_place(rows, H):
    from test_gpu_operators import BF, F32, normal, wide
    for dtype in (BF, F32):
        for pad in (0, 8):
            at = lambda t: wide(t, pad) if pad else t.clone()  # noqa: E731
            x, dy, base = normal(rows, H, dtype=dtype), normal(rows, H, seed=1, dtype=dtype), normal(rows, H, seed=2, dtype=dtype)
            w = normal(H, seed=3, dtype=dtype)
            y, mean, rstd = hap.hap_layer_norm(at(x), w)
            same = at(x)
            got = hap.hap_layer_norm(same, w, y=same)
            assert got[0] is same and torch.equal(same, y) and torch.equal(got[1], mean) and torch.equal(got[2], rstd)
            want = hap.hap_layer_norm_backward(at(dy), at(x), w, rstd, mean=mean, base=at(base))
            for which in range(3):
                t = [at(dy), at(x), at(base)]
                got = hap.hap_layer_norm_backward(t[0], t[1], w, rstd, mean=mean, base=t[2], dx=t[which])
                assert got[0] is t[which] and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_other_distances_are_refused_through_the_binding():
    x = torch.ones(6, 128, device="cuda")
    for a, b in ((x[:3, :64], x.view(12, 64)[:3]), (x.view(12, 64)[:3], x[:3, :64])):
        for call in (lambda: hap.hap_layer_norm(a, y=b), lambda: hap.hap_expert_combine(x[:, :64], torch.zeros(3, 2, dtype=torch.int32, device="cuda"), base=a, out=b)):
            with pytest.raises(hap.HapError):
                call()
    assert torch.equal(hap.hap_layer_norm(x[:1, :64], y=x.view(12, 64)[:1])[0], torch.zeros(1, 64, device="cuda"))
