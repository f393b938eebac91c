"""What the layers around RMS norm and rows in 8 bits refuse or leave behind, as far as no GPU is needed."""
import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("shape", [(7, 4, 12), (28, 12), (4, 7, 1), (1, 7, 12), (12,), (4, 7, 12, 1), (2, 14, 12)])
def test_norm_refuses_a_residual_of_another_shape(shape):
    """Matrices of as many rows in another order would be added to rows that they do not belong to."""
    from paper_1906_03707_amd import layers
    x = torch.ones(4, 7, 12)
    for a, b in ((x, torch.ones(shape)), (torch.ones(shape), x)):
        with pytest.raises(ValueError, match="residual"):
            layers.rms_norm(a, residual=b)


def test_quantized_rows_of_a_parameter_are_apart_from_it():
    from paper_1906_03707_amd import layers
    w = torch.nn.Parameter(torch.randn(5, 40, generator=torch.Generator().manual_seed(1)))
    codes, scales = layers.quantize_fp8(w)
    assert not codes.requires_grad and codes.grad_fn is None and not scales.requires_grad
    want, want_scales = layers.quantize_fp8(w.detach())
    assert torch.equal(codes.float(), want.float()) and torch.equal(scales.float(), want_scales.float())
