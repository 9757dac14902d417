"""Stacks of matrices that lie side by side, or row by row in turn, updated in place on the GPU."""
import pytest
import torch

from paper_2004_09362_amd import ar

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,M,N", [(3, 70, 90), (2, 130, 33), (4, 1, 17), (24, 64, 40)])
def test_a_fused_weight_in_place(batch, M, N, dtype):
    g = torch.Generator(device=DEV).manual_seed(M)
    x = torch.empty(batch, M, N, device=DEV).normal_(generator=g)
    w = torch.empty(batch, M, N, device=DEV).normal_(0, 0.1, generator=g).to(dtype)
    print("[gpu] fused", batch, M, N, dtype, flush=True)
    want = ar.ar_orthogonalize(x, scale=-0.1, residual=w, out_dtype=dtype)
    for gap in (0, 5):  # columns between the parts
        wide = torch.full((M, batch, N + gap), 7.0, dtype=dtype, device=DEV)
        parts = wide[:, :, :N].transpose(0, 1)
        parts.copy_(w)
        assert ar.ar_orthogonalize(x, scale=-0.1, residual=parts, out=parts).data_ptr() == wide.data_ptr()
        assert torch.equal(parts, want) and bool((wide[:, :, N:] == 7).all())
    # the update's own momentum beside each part
    both = torch.zeros(M, batch, 2, N, dtype=dtype, device=DEV)
    weights, momenta = both[:, :, 0].transpose(0, 1), both[:, :, 1].transpose(0, 1)
    weights.copy_(w)
    momenta.copy_(x)
    again = ar.ar_orthogonalize(momenta.contiguous(), scale=-0.1, residual=w, out_dtype=dtype)
    ar.ar_orthogonalize(momenta, scale=-0.1, residual=weights, out=weights)
    assert torch.equal(weights, again) and torch.equal(momenta, x.to(dtype))


def test_parts_that_share_elements_are_refused():
    wide = torch.zeros(9, 40, device=DEV)
    x = torch.ones(3, 8, 12, device=DEV)
    for bad in (wide.as_strided((3, 8, 12), (11, 40, 1)), wide.as_strided((3, 8, 12), (15, 40, 1))):  # the last: into the next row
        with pytest.raises(ar.ArError, match="y's matrices overlap"):
            ar.ar_orthogonalize(x, out=bad)
    ok = wide.as_strided((3, 8, 12), (14, 40, 1))
    ar.ar_orthogonalize(x, out=ok)
    assert torch.equal(ok, ar.ar_orthogonalize(x))
