"""Products for tests of the linear operator that reach every kernel it may launch. Which kernel a size takes is the library's choice, by estimates
that may change; so the sizes are drawn from a pool by what the library launches for them (tests/standin.py), not listed by kernel."""
import math
import random

import standin

# sizes of kernels that few sizes take: (M, K, N)
SEEN = [(5309, 64, 304), (11315, 64, 144), (5824, 704, 280), (3639, 640, 608), (1451, 832, 1520), (1984, 1280, 2392), (9256, 1472, 400), (2879, 2240, 2480), (3126, 2304, 2536), (8716, 2048, 896),
        (6592, 3456, 880), (6912, 2752, 1040), (2578, 320, 3760), (6123, 384, 1896), (5285, 1984, 2768), (3264, 704, 4448), (140, 64, 5944), (2574, 64, 8), (4053, 512, 272), (415, 1408, 8936),
        (553, 3840, 7024), (8486, 64, 8), (10429, 64, 464), (850, 64, 6816), (465, 704, 6728), (8421, 1216, 200), (883, 1472, 5000), (1157, 1792, 6352), (4351, 3008, 1872), (6257, 2368, 1152),
        (4017, 1280, 2088), (6261, 1024, 2024), (5744, 2816, 144), (395, 1280, 8944), (5267, 64, 8), (11343, 64, 8), (8665, 64, 32), (139, 2880, 416), (11, 4096, 5080), (425, 7488, 8), (519, 4032, 520),
        (11007, 384, 1440), (2148, 8768, 728), (3002, 1216, 6480), (259, 1920, 5496), (901, 6848, 1736), (1, 960, 1096), (239, 1472, 1304), (694, 448, 8584), (64, 4160, 264), (704, 768, 2896), (576, 8448, 352),
        (1024, 2240, 2320), (2624, 6208, 1192), (3264, 2112, 3192), (2624, 4288, 1856), (3456, 6912, 1152), (320, 3648, 2632), (1472, 6848, 1752), (256, 2112, 888), (64, 5760, 152), (64, 832, 2144),
        (832, 512, 4144), (1152, 8832, 472), (3200, 1344, 4840), (896, 5952, 2072), (64, 4160, 200), (320, 640, 2840), (5760, 2560, 1568), (640, 192, 392), (1063, 64, 240), (637, 512, 400), (812, 5312, 304),
        (12, 576, 6624), (64, 4672, 1136), (20, 6016, 8), (33, 2880, 8), (1, 4160, 8), (1, 8384, 16), (198, 13440, 2392), (64, 4096, 768)]


def pool():
    rng = random.Random(59)
    log = lambda low, high: math.exp(rng.uniform(math.log(low), math.log(high)))  # noqa: E731
    sizes = list(SEEN)
    while len(sizes) < 1500:
        M, K, N = int(log(1, 12000)), max(64, int(log(64, 9000)) // 64 * 64), int(log(8, 9000)) // 8 * 8
        if rng.random() < 0.5:
            M = max(64, M // 64 * 64)
        if M * K * N <= 3e10:
            sizes.append((M, K, N))
    return [dict(op=op, fields=dict(M=M, K=K, N=N, weight_layout=nk, activation=4)) for M, K, N in sizes for nk in (0, 1) for op in ("linear", "linear_backward")]


def of_the_operator(kernel):
    return kernel.startswith(("linear_", "turn_kernel<4", "sum_rows")) or "WithEpilogue" in kernel


def reached(lib):
    """{kernel: the calls that launch it} for the linear operator's kernels, its own and those of the plain product that it calls."""
    calls = pool()
    out, kernels = standin.run(lib, calls)
    by = {k: [] for k in kernels if of_the_operator(k) or k.startswith("gemm_blocks_kernel")}
    for call, r in zip(calls, out):
        assert r["status"] == 0, call
        for kernel in {l.kernel for l in r["launches"]}:
            if kernel in by:
                by[kernel].append(call)
    return by


def picked(by):
    """A few calls of each kernel, (op, M, K, N, weight_layout): the smallest, and the smallest whose rows and columns fill no tile."""
    out = {}
    for calls in by.values():
        size = lambda c: c["fields"]["M"] * c["fields"]["K"] * c["fields"]["N"]  # noqa: E731
        odd = lambda c: (c["fields"]["M"] % 64 == 0) + (c["fields"]["N"] % 64 == 0)  # noqa: E731
        for best in (sorted(calls, key=size)[:1], sorted(calls, key=lambda c: (odd(c), size(c)))[:2]):
            for c in best:
                f = c["fields"]
                out[c["op"], f["M"], f["K"], f["N"], f["weight_layout"]] = None
    return list(out)
