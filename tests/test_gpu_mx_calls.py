"""Calls as the binding takes them: sizes that do not fit, memory that runs out, and the memory of what a call makes for a given stream."""
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


def test_memory_that_runs_out(tq):
    """The error is torch's own for that, which programs catch to make room."""
    for call in (lambda: tq.new_mx(2 ** 31 - 1, 2 ** 24), lambda: tq.tq_mx_product(*[tq.MxMatrix(None, None, 2 ** 21, 0, memory=ones(1).byte())] * 2, torch.float32)):
        with pytest.raises(torch.OutOfMemoryError):
            call()


# ---- a stream given by hand: what the call makes is that stream's memory -------------------------------------------------
def pool_of(t):
    """The stream whose memory a tensor lies in."""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not in the allocator's memory")


def calls(tq):
    """Every call that makes its outputs, as a function of the stream; the inputs are ready."""
    g = torch.randn(3, 4096, device="cuda") * 1e-3
    stats = tq.tq_stats(g)
    params = [tq.tq_params(s, 16, tq.NONUNIFORM, gamma=3.0) for s in tq.stats_to_host(stats)]
    params_dev = tq.tq_params_device(stats, 3, 16, tq.NONUNIFORM, 3.0)
    packed = tq.tq_compress(g, params, seed=1)
    groups = [(0, 1024), (1024, 2000)]
    group_params = tq.tq_params_device(tq.tq_stats_segments(g, groups), 6, 16, tq.NONUNIFORM, 3.0)
    x, m = torch.randn(64, 96, device="cuda"), tq.tq_mx_quantize(torch.randn(64, 96, device="cuda"))
    rows, gu = tq.tq_mx_quantize(g, layout=tq.MX_ROWS), torch.randn(64, 192, device="cuda")

    def hint(n):
        h = tq.new_gmin_hint(n)
        torch.cuda.synchronize()
        return h
    torch.cuda.synchronize()
    return dict(
        stats=lambda s: tq.tq_stats(g, stream=s),
        stats_hinted=lambda s: tq.tq_stats_hinted(g, hint(3), stream=s),
        stats_segments=lambda s: tq.tq_stats_segments(g, groups, stream=s),
        stats_hinted_segments=lambda s: tq.tq_stats_hinted_segments(g, groups, hint(6), stream=s),
        params_device=lambda s: tq.tq_params_device(stats, 3, 16, tq.NONUNIFORM, 3.0, stream=s),
        compress=lambda s: tq.tq_compress(g, params, seed=1, stream=s),
        compress_device_params=lambda s: tq.tq_compress_device_params(g, params_dev, 16, tq.NONUNIFORM, 1, stream=s),
        compress_segments=lambda s: tq.tq_compress_segments(g, groups, group_params, 16, tq.NONUNIFORM, 1, stream=s),
        aggregate=lambda s: tq.tq_decompress_aggregate(packed, 4096, params, stream=s),
        aggregate_rows=lambda s: tq.tq_decompress_aggregate_rows(list(packed), 4096, params, stream=s),
        aggregate_device_params=lambda s: tq.tq_decompress_aggregate_device_params(packed, 4096, params_dev, 16, stream=s),
        mx_quantize=lambda s: tq.tq_mx_quantize(x, stream=s),
        mx_quantize_both=lambda s: tq.tq_mx_quantize_both(x, stream=s),
        mx_dequantize=lambda s: tq.tq_mx_dequantize(m, stream=s),
        mx_decompress_aggregate=lambda s: tq.tq_mx_decompress_aggregate(rows, stream=s),
        mx_product=lambda s: tq.tq_mx_product(m, m, stream=s),
        mx_gated=lambda s: tq.tq_mx_gated(m, m, m, stream=s),
        mx_gated_backward=lambda s: tq.tq_mx_gated_backward(x, gu, stream=s),
    )


def tensors(result):
    return [t.memory if hasattr(t, "memory") else t for t in (result if isinstance(result, tuple) else (result,))]


def test_results_are_memory_of_the_given_stream(tq):
    for name, call in calls(tq).items():
        stream = torch.cuda.Stream()
        want = [t.clone() for t in tensors(call(None))]
        torch.cuda.synchronize()
        for given in (stream, stream.cuda_stream):                     # an object, a handle
            got = tensors(call(given))
            torch.cuda.synchronize()
            for t, w in zip(got, want, strict=True):
                assert pool_of(t) == stream.cuda_stream, name
                if not name.startswith("mx"):                          # what lies between a matrix's rows is not written
                    assert torch.equal(t, w), name
        current = torch.cuda.current_stream()
        for given in (None, current, current.cuda_stream):
            got = tensors(call(given))
            torch.cuda.synchronize()
            assert all(pool_of(t) == current.cuda_stream for t in got), name


def test_handles_of_the_default_streams(tq):
    """0 and 1 are the legacy default stream, 2 is the thread's own: CUDA's names for them, taken by every call and from every current stream."""
    for name, call in calls(tq).items():
        want = [t.clone() for t in tensors(call(None))]
        torch.cuda.synchronize()
        for current in (torch.cuda.default_stream(), torch.cuda.Stream()):
            with torch.cuda.stream(current):
                for handle in (0, 1, 2):
                    got = tensors(call(handle))
                    torch.cuda.synchronize()
                    for t, w in zip(got, want, strict=True):
                        assert pool_of(t) == (2 if handle == 2 else 0), (name, handle)
                        if not name.startswith("mx"):
                            assert torch.equal(t, w), (name, handle)


def test_memory_in_use_on_the_current_stream_is_left_alone(tq):
    """A block that the current stream frees while a slow kernel there has yet to read it: a call on another stream takes none of it."""
    m = tq.tq_mx_quantize(torch.randn(1024, 1024, device="cuda"))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        a = torch.full((1024, 1024), 7.0, device="cuda")
        into = torch.zeros_like(a)
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)                                  # some 10 ms
        into.copy_(a)
        del a
        out = tq.tq_mx_dequantize(m, stream=stream)
        torch.cuda.synchronize()
        assert (into == 7).all()
        del out


def test_results_dropped_on_the_current_stream(tq):
    """Used there after the given stream, and dropped while that use is still to come: the given stream's next call takes other memory."""
    m = tq.tq_mx_quantize(torch.randn(1024, 1024, device="cuda"))
    want = tq.tq_mx_dequantize(m)
    other = tq.tq_mx_quantize(torch.zeros(1024, 1024, device="cuda"))
    into, stream = torch.empty_like(want), torch.cuda.Stream()
    torch.cuda.synchronize()
    out = tq.tq_mx_dequantize(m, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda._sleep(20_000_000)
    into.copy_(out)
    at = out.data_ptr()
    del out
    again = tq.tq_mx_dequantize(other, stream=stream)
    assert again.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(into, want)


def test_streams_by_hand_inside_a_graph(tq):
    """A call on a forked stream of a capture makes its outputs in the graph's memory."""
    m = tq.tq_mx_quantize(torch.randn(64, 96, device="cuda"))
    want = tq.tq_mx_product(m, m)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = tq.tq_mx_product(m, m, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        twice = out + out
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(twice, want + want)


def test_longest_sums(tq):
    """Sums of close to 2^31 products: the wait for the whole of one lasts as long as its stages are filled.  All are ones, so that every partial sum is exact."""
    k = 2 ** 31 - 256
    ones_of = lambda rows, k: tq.MxMatrix(torch.full((rows, k // 2), 0x22, dtype=torch.uint8, device="cuda"),  # noqa: E731
                                          torch.full((-(-rows // 128), k // 128 * 512), 127, dtype=torch.uint8, device="cuda"), rows, k)
    a = ones_of(1, k)
    assert tq.tq_mx_product(a, a, torch.float32).item() == k
    assert tq.tq_wait_expired_count() == 0
    del a
    k = 2 ** 27 - 256
    a, b = ones_of(130, k), ones_of(3, k)
    assert (tq.tq_mx_product(a, b, torch.float32) == k).all()
    del a, b
    torch.cuda.empty_cache()
