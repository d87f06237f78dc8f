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
