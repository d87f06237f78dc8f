"""What a layer of experts launches, on the host."""
import launch_log


def test_a_function_attribute_does_not_depend_on_the_call():
    """It belongs to the function and the device: a call that set less than another thread's launch takes could come between that one's
    attribute and its launch."""
    calls = [[name, rows, N, K, groups] for groups in (1, 64, 1024) for name, rows, N, K in
             (("gemm", 30000, 4096, 1024), ("gemm", 6000, 512, 512), ("wgrad", 30000, 4096, 1024), ("wgrad", 2048, 256, 300))]
    values, most = {}, {}
    for r in launch_log.record(calls):
        assert r["status"] == 0
        for kernel, what, value in r["attributes"]:
            values.setdefault((kernel, what), set()).add(value)
        for kernel, _, _, lds in r["launches"]:
            most[kernel] = max(most.get(kernel, 0), lds)
    assert len(values) == 4, values    # both tiles, forward and weight gradient
    for (kernel, _), v in values.items():
        assert len(v) == 1 and max(v) >= most[kernel], (kernel, v, most[kernel])


def test_rows_that_are_read_again_are_not_read_past_the_cache():
    """The quantization passes the last-level cache by where the source is larger, not where a small source is gathered many times over."""
    sizes = [(131072, 1024, 64, 0), (131072, 1024, 64, 16384), (131072, 1024, 64, 131072), (131072, 1024, 64, 1 << 20), (131071, 1024, 64, 1 << 20), (131072, 1021, 64, 0)]
    for along, turned in ((1, 0), (0, 1), (1, 1)):
        past = [r["launches"][0][0].split("<")[1].rstrip(">").split(", ")[-1] for r in launch_log.record([["quantize", *s, along, turned] for s in sizes])]
        assert past == ["true", "false", "true", "true", "false", "false"], (along, turned)
