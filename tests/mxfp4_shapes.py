"""Products (M, N, K, batch) that reach each kernel form of loka_mxfp4_gemm; tests/test_mxfp4_forms.py holds them to it."""
STREAM, LARGE, HALVES, SMALL = range(4)
SPLIT = "split"          # HALVES with a contraction split over workgroups

SHAPES = {
    STREAM: [(5, 130, 700, 1), (40, 300, 1030, 3)],
    LARGE: [(4096, 4096, 640, 1), (4090, 4083, 700, 1), (1010, 1001, 516, 16), (1010, 1008, 516, 16)],
    HALVES: [(2048, 2048, 4096, 1), (2045, 2043, 4100, 1), (500, 511, 4100, 8), (512, 256, 4000, 16)],
    SMALL: [(2048, 2048, 640, 1), (2040, 2033, 700, 1), (520, 392, 300, 8), (700, 515, 300, 40), (9001, 1025, 256, 1)],
    SPLIT: [(300, 1024, 16384, 1), (515, 516, 16500, 1), (520, 516, 8320, 2), (257, 385, 16640, 3)],
}
ALL = [(form, *s) for form, shapes in SHAPES.items() for s in shapes]
