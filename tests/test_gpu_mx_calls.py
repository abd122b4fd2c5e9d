"""Calls of the microscaled 4-bit operators as the binding takes them: sizes that do not fit, streams, memory that runs out."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2402_01798_b200 import binding
    binding.lib()
    yield binding
    assert binding.tq_wait_expired_count() == 0


def ones(*size):
    return torch.ones(size, device="cuda")


def test_sizes_have_to_fit(tq):
    """A tensor that is larger than its call is refused like one that is smaller: nothing says which part is meant."""
    x, m, small = ones(64, 96), tq.tq_mx_quantize(ones(64, 96)), tq.tq_mx_quantize(ones(32, 64))
    refused = [
        lambda: tq.tq_mx_quantize(x, out=tq.new_mx(63, 96)),
        lambda: tq.tq_mx_quantize(x, out=tq.new_mx(64, 95)),
        lambda: tq.tq_mx_quantize(x, out=tq.new_mx(64, 97)),
        lambda: tq.tq_mx_quantize(x, cols=64, out=tq.new_mx(64, 96)),
        lambda: tq.tq_mx_quantize(x, cols=64, out=tq.new_mx(64, 32)),
        lambda: tq.tq_mx_quantize(x[0], out=tq.new_mx(1, 64)),
        lambda: tq.tq_mx_quantize_both(x, out=tq.new_mx(32, 96), out_t=tq.new_mx(96, 32)),
        lambda: tq.tq_mx_quantize_both(x, out=tq.new_mx(64, 64), out_t=tq.new_mx(64, 64)),
        lambda: tq.tq_mx_dequantize(m, out=ones(65, 96)),
        lambda: tq.tq_mx_dequantize(m, out=ones(64, 97)),
        lambda: tq.tq_mx_decompress_aggregate(tq.tq_mx_quantize(x, layout=tq.MX_ROWS), out=ones(2, 96)),
        lambda: tq.tq_mx_product(m, m, out=ones(64, 65)),
        lambda: tq.tq_mx_product(m, m, out=ones(65, 64)),
        lambda: tq.tq_mx_gated(small, small, small, projections=ones(32, 65)),
        lambda: tq.tq_mx_gated(small, small, small, projections=ones(33, 64)),
        lambda: tq.tq_mx_gated_backward(ones(4, 32), ones(4, 128)),            # u would come from g's columns
        lambda: tq.tq_mx_gated_backward(ones(4, 32), ones(5, 64)),
        lambda: tq.tq_mx_gated_backward(ones(5, 32), ones(4, 64)),
        lambda: tq.tq_mx_gated_backward(ones(4, 64), ones(4, 64), dgu=tq.new_mx(4, 64), dgu_t=tq.new_mx(64, 4), h_t=tq.new_mx(32, 4)),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(ValueError, match="larger|smaller|columns"):
            call()
            pytest.fail(f"call {i} was taken")


def test_parts_of_larger_tensors_are_taken(tq):
    """What is meant is passed as a view; messages and their mean also have a form without one."""
    x = torch.randn(64, 104, device="cuda")
    part = tq.tq_mx_quantize(x[:, :96].contiguous())
    assert torch.equal(tq.tq_mx_quantize(x[:, :96]).codes, part.codes)
    assert torch.equal(tq.tq_mx_quantize(x, cols=96).codes, part.codes)
    assert torch.equal(tq.tq_mx_quantize(x, cols=96, out=tq.new_mx(64, 96)).scales, part.scales)
    rows = tq.tq_mx_quantize(x, cols=96, layout=tq.MX_ROWS)
    out = torch.full((104,), -7.0, device="cuda")
    tq.tq_mx_decompress_aggregate(rows, out=out)
    assert torch.equal(out[:96], tq.tq_mx_decompress_aggregate(rows)) and (out[96:] == -7).all()
