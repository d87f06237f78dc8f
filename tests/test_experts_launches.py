"""What a layer of experts launches, on the host."""
import launch_log
import test_gpu_experts as G
import test_gpu_experts_mended as M


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


# what each of test_gpu_experts.FORMS runs, so that a changed choice cannot leave a form untested
SMALL, LARGE = "gg_tile_kernel<GgTile<4, 4, 2, 2>, false>", "gg_tile_kernel<GgTile<8, 4, 2, 4>, false>"
ROWS16 = {n: "gg_stream_kernel<1, %d, " % n for n in (1, 2, 4)}        # 16 rows at a time: the linear quantizes inside
ROWS32 = "gg_stream_kernel<2, 4, false>"
FORM_OF = [ROWS16[4], ROWS16[2], ROWS16[2], ROWS16[1], ROWS32, ROWS32, SMALL, SMALL, SMALL, SMALL, LARGE, LARGE, LARGE, SMALL, LARGE, SMALL, LARGE]


def test_the_tested_products_reach_their_forms():
    assert len(FORM_OF) == len(G.FORMS) and {*ROWS16.values(), ROWS32, SMALL, LARGE} == set(FORM_OF)
    calls = [[op, sum(sizes) + 19, N, K, len(sizes), turned] for sizes, K, N in G.FORMS for turned in (1, 0) for op in ("gemm", "linear")]
    got = launch_log.record(calls)
    for i, want in enumerate(FORM_OF):
        for call, r in zip(calls[4 * i:4 * i + 4], got[4 * i:4 * i + 4]):
            names = [l[0] for l in r["launches"]]
            if want.endswith(">"):     # of stored operands; the linear quantizes before
                assert names[-1] == want and [n.split("<")[0] for n in names[:-1]] == (["gq_along_kernel"] if call[0] == "linear" else []), call
            else:
                assert names == [want + ("true>" if call[0] == "linear" else "false>")], call


def _cases(test):
    return [m.args[1] for m in test.pytestmark if m.name == "parametrize"]


def test_the_tested_weight_gradients_reach_their_forms():
    """Partial sums, and both tiles in several rounds of workgroups: up to 64 groups (the longest first) and above."""
    small, large = SMALL.replace("false", "true"), LARGE.replace("false", "true")
    uneven = _cases(G.test_weight_gradients_of_many_uneven_groups)[0] + _cases(M.test_weight_gradients_of_many_groups)[0]
    got = launch_log.record([["wgrad", sum(sizes) + 9, 720, 1008, len(sizes)] for sizes in uneven])
    assert [(len(sizes) <= 64, r["launches"][0][0]) for sizes, r in zip(uneven, got)] == [(True, small), (True, large), (False, small), (True, large), (False, large)]
    for sizes, r in zip(uneven, got):
        rows, cols = (256, 256) if r["launches"][0][0] == large else (128, 128)
        assert len(r["launches"]) == 1 and -(-1008 // rows) * -(-720 // cols) * len(sizes) > r["launches"][0][1]       # several rounds
    sizes = _cases(G.test_weight_gradients_are_exact_on_whole_numbers)
    split = launch_log.record([["wgrad", sum(s) + 9, N, K, len(s)] for s in sizes[0] for K, N in sizes[1]])
    assert sum([l[0] for l in r["launches"]] == [small, "gg_join_kernel"] for r in split) >= 4


def test_the_tested_choices_reach_their_forms():
    """Chunks of each size, their counts added up in the placing kernel (in one round of loads and in several) and by a launch of its own, every
    number of lanes and logits in both."""
    cases = _cases(M.test_route_sizes)[0]
    reached, rounds = {}, set()
    for (T, E, k, score, renorm, bf16), r in zip(cases, launch_log.record([["route", T, E, k, bf16] for T, E, k, _, _, bf16 in cases])):
        names = [l[0] for l in r["launches"]]
        chunks = r["launches"][0][1]
        scanned = "route_scan_kernel" in names
        assert names[1:] == (["route_scan_kernel", "route_place_kernel<true>"] if scanned else ["route_place_kernel<false>"])
        chunk = next(c for c in (16, 32, 64, 128) if -(-T // c) == chunks)
        reached.setdefault((chunk, scanned), set()).add(names[0].split("<")[1].split(", ")[0:2][0] + " x " + names[0].split(", ")[1])
        pitch = max(4, 1 << (E - 1).bit_length())
        rounds.add(scanned or chunks > 8 * (1024 // (pitch // 4)))
    assert set(reached) == {(16, False), (32, False), (64, False), (128, False), (128, True)} and rounds == {False, True}
    every = {"16 x 4", "16 x 8", "16 x 16", "64 x 8", "64 x 16"}
    assert reached[(128, True)] == every and reached[(128, False)] | reached[(64, False)] | reached[(32, False)] == every, reached
