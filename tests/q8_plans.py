"""Products that reach every kernel of the 8-bit product, in every way that its rule of sizes launches
one: whole tiles, all of them split over K, the last round's split; columns of tiles that start at other places of K;
rows off lines of 128 bytes, where a kernel has a form for them; K past the last whole step.

The rule is asked on the host (q8_plan_check.cpp): test_q8_plans_cpu.py holds CASES to the launches that they are named by,
and to all that a sample of sizes, strides and workspaces reaches."""
import os
import shutil
import subprocess

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)

# name, bytes of K a step, whether rows off lines have a kernel of their own; in the rule's order
KERNELS = [("few 4 waves", 256, False), ("few 8 waves", 256, False), ("ring 32x32", 256, False), ("ring 32x64", 256, True),
           ("ring 64x64", 256, False), ("ring 64x128", 128, True), ("ring 128x64", 256, False), ("ring 128x128", 128, True),
           ("wide 128x256", 128, True), ("wide 192x256", 128, False), ("wide 256x256", 128, False)]
TILES = [(16, 16), (16, 16), (32, 32), (32, 64), (64, 64), (64, 128), (128, 64), (128, 128), (128, 256), (192, 256), (256, 256)]
ASKED = 64 << 20  # a workspace that any launch fits in

# kernel, launch, (M, N, K, row strides of X and W, bytes from a line of 128 to X and to W, workspace)
CASES = [
    ("few 4 waves", "whole", (8, 12415, 256, 256, 256, 0, 0, ASKED)),
    ("few 4 waves", "whole, rest", (1, 12303, 16, 16, 16, 0, 0, 0)),
    ("few 8 waves", "whole", (8, 65, 256, 352, 288, 64, 80, 0)),
    ("few 8 waves", "whole, rest", (8, 65, 16, 160, 192, 96, 32, ASKED)),
    ("ring 32x32", "last round split", (30, 16746, 5120, 5184, 5152, 64, 32, ASKED)),
    ("ring 32x32", "last round split, rest", (24, 16489, 5040, 5040, 5040, 0, 0, ASKED)),
    ("ring 32x32", "last round split, starts apart", (8, 17093, 8192, 8192, 8192, 0, 0, 572401)),
    ("ring 32x32", "last round split, starts apart, rest", (57, 8448, 36768, 36864, 36864, 0, 0, 1352472)),
    ("ring 32x32", "split", (19, 133, 3072, 3152, 3072, 16, 112, ASKED)),
    ("ring 32x32", "split past 8", (10, 133, 6400, 6416, 6416, 112, 16, ASKED)),
    ("ring 32x32", "split past 8, rest", (9, 134, 6192, 6192, 6192, 0, 0, ASKED)),
    ("ring 32x32", "split past 8, starts apart", (9, 545, 8192, 8192, 8192, 0, 0, ASKED)),
    ("ring 32x32", "split past 8, starts apart, rest", (13, 715, 8176, 8192, 8192, 0, 0, ASKED)),
    ("ring 32x32", "split, rest", (20, 138, 3216, 3216, 3216, 0, 0, ASKED)),
    ("ring 32x32", "split, starts apart", (19, 545, 4096, 4096, 4096, 0, 0, ASKED)),
    ("ring 32x32", "split, starts apart, rest", (17, 550, 4080, 4096, 4096, 0, 0, ASKED)),
    ("ring 32x32", "whole", (17, 129, 256, 256, 256, 0, 0, ASKED)),
    ("ring 32x32", "whole, rest", (17, 129, 16, 128, 224, 64, 16, ASKED)),
    ("ring 32x32", "whole, starts apart", (17, 545, 4096, 4096, 4096, 0, 0, 0)),
    ("ring 32x32", "whole, starts apart, rest", (51, 597, 3984, 4096, 4096, 0, 0, 0)),
    ("ring 32x64", "last round split", (11, 16986, 6144, 6144, 6144, 0, 0, ASKED)),
    ("ring 32x64", "last round split, off lines", (13, 17818, 7936, 7968, 7968, 96, 32, ASKED)),
    ("ring 32x64", "last round split, off lines, rest", (29, 18070, 6336, 6336, 6336, 0, 0, ASKED)),
    ("ring 32x64", "last round split, rest", (8, 16741, 5872, 5888, 5888, 0, 0, ASKED)),
    ("ring 32x64", "last round split, starts apart", (12, 16434, 8192, 8192, 8192, 0, 0, ASKED)),
    ("ring 32x64", "last round split, starts apart, rest", (21, 17146, 8160, 8192, 8192, 0, 0, ASKED)),
    ("ring 32x64", "split", (33, 915, 5632, 5632, 5632, 0, 0, ASKED)),
    ("ring 32x64", "split past 8", (44, 635, 6144, 6144, 6144, 0, 0, ASKED)),
    ("ring 32x64", "split past 8, off lines", (13, 865, 8192, 8224, 8192, 32, 0, ASKED)),
    ("ring 32x64", "split past 8, off lines, rest", (21, 886, 8240, 8240, 8240, 0, 0, ASKED)),
    ("ring 32x64", "split past 8, rest", (33, 419, 8336, 8448, 8448, 0, 0, ASKED)),
    ("ring 32x64", "split past 8, starts apart", (9, 1097, 8192, 8192, 8192, 0, 0, ASKED)),
    ("ring 32x64", "split past 8, starts apart, rest", (3, 1193, 8144, 8192, 8192, 0, 0, ASKED)),
    ("ring 32x64", "split, off lines", (21, 1761, 4096, 4160, 4096, 16, 0, ASKED)),
    ("ring 32x64", "split, off lines, rest", (17, 1843, 4208, 4320, 4304, 96, 112, ASKED)),
    ("ring 32x64", "split, rest", (51, 869, 4240, 4352, 4352, 0, 0, ASKED)),
    ("ring 32x64", "split, starts apart", (19, 1446, 4096, 4096, 4096, 0, 0, ASKED)),
    ("ring 32x64", "split, starts apart, rest", (25, 1570, 8112, 8192, 8192, 0, 0, ASKED)),
    ("ring 32x64", "whole", (8, 14722, 1280, 1280, 1280, 0, 0, ASKED)),
    ("ring 32x64", "whole, rest", (13, 16345, 1008, 1024, 1024, 0, 0, ASKED)),
    ("ring 32x64", "whole, starts apart", (11, 9725, 4096, 4096, 4096, 0, 0, ASKED)),
    ("ring 32x64", "whole, starts apart, rest", (23, 9743, 4000, 4096, 4096, 0, 0, ASKED)),
    ("ring 64x64", "last round split", (407, 2458, 14848, 14848, 14848, 0, 0, 4712795)),
    ("ring 64x64", "last round split, rest", (305, 3429, 10432, 10496, 10496, 0, 0, 10561818)),
    ("ring 64x64", "last round split, starts apart", (78, 8393, 12288, 12288, 12288, 0, 0, 7472301)),
    ("ring 64x64", "last round split, starts apart, rest", (46, 16467, 8080, 8192, 8192, 0, 0, ASKED)),
    ("ring 64x64", "split", (205, 258, 4096, 4096, 4096, 0, 0, ASKED)),
    ("ring 64x64", "split past 8", (140, 265, 6144, 6144, 6144, 0, 0, ASKED)),
    ("ring 64x64", "split past 8, rest", (68, 343, 6320, 6496, 6448, 112, 112, ASKED)),
    ("ring 64x64", "split past 8, starts apart", (70, 257, 8192, 8192, 8192, 0, 0, ASKED)),
    ("ring 64x64", "split past 8, starts apart, rest", (70, 325, 12272, 12288, 12288, 0, 0, ASKED)),
    ("ring 64x64", "split, rest", (325, 285, 2576, 2688, 2688, 0, 0, ASKED)),
    ("ring 64x64", "split, starts apart", (72, 1307, 4096, 4096, 4096, 0, 0, ASKED)),
    ("ring 64x64", "split, starts apart, rest", (86, 1213, 3984, 4096, 4096, 0, 0, ASKED)),
    ("ring 64x64", "whole", (65, 262, 512, 512, 512, 0, 0, ASKED)),
    ("ring 64x64", "whole, rest", (66, 267, 144, 256, 256, 0, 0, 0)),
    ("ring 64x64", "whole, starts apart", (66, 1114, 4096, 4096, 4096, 0, 0, 0)),
    ("ring 64x64", "whole, starts apart, rest", (67, 1142, 4080, 4096, 4096, 0, 0, 0)),
    ("ring 64x128", "last round split", (421, 4864, 7040, 7040, 7040, 0, 0, ASKED)),
    ("ring 64x128", "last round split, off lines", (478, 4121, 7040, 7088, 7088, 80, 0, ASKED)),
    ("ring 64x128", "last round split, off lines, rest", (463, 4213, 7184, 7360, 7376, 112, 112, ASKED)),
    ("ring 64x128", "last round split, rest", (16, 33331, 1840, 1920, 1920, 0, 0, ASKED)),
    ("ring 64x128", "split", (69, 514, 1920, 1920, 1920, 0, 0, ASKED)),
    ("ring 64x128", "split past 8", (75, 517, 3200, 3200, 3200, 0, 0, ASKED)),
    ("ring 64x128", "split past 8, off lines", (71, 578, 3072, 3152, 3184, 0, 16, ASKED)),
    ("ring 64x128", "split past 8, off lines, rest", (82, 530, 3120, 3216, 3232, 0, 0, ASKED)),
    ("ring 64x128", "split past 8, rest", (77, 586, 3088, 3200, 3200, 0, 0, ASKED)),
    ("ring 64x128", "split, off lines", (74, 530, 1920, 2032, 1936, 64, 80, ASKED)),
    ("ring 64x128", "split, off lines, rest", (82, 518, 1824, 1824, 1824, 0, 0, ASKED)),
    ("ring 64x128", "split, rest", (65, 601, 2128, 2176, 2176, 0, 0, ASKED)),
    ("ring 64x128", "whole", (69, 514, 128, 128, 128, 0, 0, 0)),
    ("ring 64x128", "whole, off lines", (69, 531, 128, 128, 128, 64, 16, 0)),
    ("ring 64x128", "whole, off lines, rest", (65, 513, 16, 16, 16, 0, 0, ASKED)),
    ("ring 64x128", "whole, rest", (68, 513, 16, 128, 128, 0, 0, 0)),
    ("ring 128x64", "last round split", (3759, 524, 9984, 10048, 10080, 96, 96, ASKED)),
    ("ring 128x64", "last round split, rest", (5629, 383, 9776, 9888, 9936, 48, 64, ASKED)),
    ("ring 128x64", "last round split, starts apart", (82, 16689, 8192, 8192, 8192, 0, 0, ASKED)),
    ("ring 128x64", "last round split, starts apart, rest", (91, 17280, 8096, 8192, 8192, 0, 0, ASKED)),
    ("ring 128x64", "split", (569, 257, 2048, 2048, 2048, 0, 0, ASKED)),
    ("ring 128x64", "split past 8", (514, 256, 6144, 6144, 6144, 0, 0, ASKED)),
    ("ring 128x64", "split past 8, rest", (523, 256, 6240, 6272, 6272, 0, 0, ASKED)),
    ("ring 128x64", "split past 8, starts apart", (87, 1311, 20480, 20480, 20480, 0, 0, ASKED)),
    ("ring 128x64", "split past 8, starts apart, rest", (104, 1280, 53152, 53248, 53248, 0, 0, ASKED)),
    ("ring 128x64", "split, rest", (528, 265, 2688, 2688, 2688, 0, 0, ASKED)),
    ("ring 128x64", "split, starts apart", (83, 3201, 8192, 8192, 8192, 0, 0, ASKED)),
    ("ring 128x64", "split, starts apart, rest", (102, 3456, 12192, 12288, 12288, 0, 0, ASKED)),
    ("ring 128x64", "whole", (517, 266, 256, 256, 256, 0, 0, ASKED)),
    ("ring 128x64", "whole, rest", (544, 258, 192, 192, 192, 0, 0, 0)),
    ("ring 128x64", "whole, starts apart", (66, 10327, 4096, 4096, 4096, 0, 0, 0)),
    ("ring 128x64", "whole, starts apart, rest", (76, 9265, 4080, 4096, 4096, 0, 0, ASKED)),
    ("ring 128x128", "last round split", (1743, 2331, 4864, 4864, 4864, 0, 0, ASKED)),
    ("ring 128x128", "last round split, off lines", (1430, 2785, 3328, 3392, 3392, 32, 0, ASKED)),
    ("ring 128x128", "last round split, off lines, rest", (2252, 1855, 3040, 3040, 3040, 0, 0, ASKED)),
    ("ring 128x128", "last round split, rest", (1987, 2087, 6112, 6144, 6144, 0, 0, ASKED)),
    ("ring 128x128", "split", (513, 1, 1920, 1920, 1920, 0, 0, ASKED)),
    ("ring 128x128", "split past 8", (522, 2, 3712, 3712, 3712, 0, 0, ASKED)),
    ("ring 128x128", "split past 8, off lines", (527, 5, 3456, 3552, 3520, 80, 112, ASKED)),
    ("ring 128x128", "split past 8, off lines, rest", (517, 78, 3440, 3440, 3440, 0, 0, ASKED)),
    ("ring 128x128", "split past 8, rest", (250, 657, 28864, 28928, 28928, 0, 0, ASKED)),
    ("ring 128x128", "split, off lines", (532, 2, 1792, 1904, 1888, 112, 80, ASKED)),
    ("ring 128x128", "split, off lines, rest", (525, 2, 1824, 2016, 2000, 80, 112, ASKED)),
    ("ring 128x128", "split, rest", (528, 1183, 4432, 4480, 4480, 0, 0, ASKED)),
    ("ring 128x128", "whole", (520, 542, 128, 128, 128, 0, 0, 0)),
    ("ring 128x128", "whole, off lines", (554, 515, 128, 160, 144, 48, 0, 0)),
    ("ring 128x128", "whole, off lines, rest", (526, 514, 32, 160, 128, 0, 112, ASKED)),
    ("ring 128x128", "whole, rest", (529, 515, 32, 128, 128, 0, 0, 0)),
    ("wide 128x256", "last round split", (3673, 2097, 12288, 12288, 12288, 0, 0, ASKED)),
    ("wide 128x256", "last round split, off lines", (3671, 2209, 4608, 4704, 4720, 0, 32, ASKED)),
    ("wide 128x256", "last round split, off lines, rest", (2417, 3447, 6976, 6976, 6976, 0, 0, ASKED)),
    ("wide 128x256", "last round split, rest", (2778, 2835, 15184, 15232, 15232, 0, 0, ASKED)),
    ("wide 128x256", "split", (1100, 1165, 8192, 8192, 8192, 0, 0, ASKED)),
    ("wide 128x256", "split past 8", (378, 1050, 73728, 73728, 73728, 0, 0, ASKED)),
    ("wide 128x256", "split past 8, off lines", (552, 1024, 68352, 68400, 68432, 32, 80, ASKED)),
    ("wide 128x256", "split past 8, off lines, rest", (462, 1034, 80704, 80784, 80768, 112, 16, ASKED)),
    ("wide 128x256", "split past 8, rest", (254, 1346, 59040, 59136, 59136, 0, 0, ASKED)),
    ("wide 128x256", "split, off lines", (1180, 1142, 11136, 11248, 11152, 48, 80, ASKED)),
    ("wide 128x256", "split, off lines, rest", (1052, 1798, 6832, 6944, 6960, 16, 32, ASKED)),
    ("wide 128x256", "split, rest", (953, 1342, 11552, 11648, 11648, 0, 0, ASKED)),
    ("wide 128x256", "whole", (132, 16629, 128, 128, 128, 0, 0, 0)),
    ("wide 128x256", "whole, off lines", (129, 23169, 128, 144, 176, 16, 96, 0)),
    ("wide 128x256", "whole, off lines, rest", (137, 22381, 176, 176, 176, 0, 0, 0)),
    ("wide 128x256", "whole, rest", (141, 16953, 144, 256, 256, 0, 0, ASKED)),
    ("wide 192x256", "last round split", (567, 21983, 2304, 2304, 2304, 0, 0, ASKED)),
    ("wide 192x256", "last round split, rest", (518, 21785, 3184, 3248, 3216, 0, 112, ASKED)),
    ("wide 192x256", "split", (518, 3267, 8192, 8192, 8192, 0, 0, ASKED)),
    ("wide 192x256", "split past 8", (553, 1602, 18560, 18560, 18560, 0, 0, ASKED)),
    ("wide 192x256", "split past 8, rest", (560, 1577, 22208, 22272, 22272, 0, 0, ASKED)),
    ("wide 192x256", "split, rest", (906, 2207, 11216, 11264, 11264, 0, 0, ASKED)),
    ("wide 192x256", "whole", (259, 22067, 128, 128, 128, 0, 0, ASKED)),
    ("wide 192x256", "whole, rest", (261, 22414, 176, 256, 256, 0, 0, 0)),
    ("wide 256x256", "last round split", (1740, 9226, 1920, 1920, 1920, 0, 0, ASKED)),
    ("wide 256x256", "last round split, rest", (2505, 6617, 1712, 1808, 1824, 32, 48, ASKED)),
    ("wide 256x256", "split", (2013, 1399, 10880, 10880, 10880, 0, 0, ASKED)),
    ("wide 256x256", "split past 8", (388, 2063, 24576, 24576, 24576, 0, 0, ASKED)),
    ("wide 256x256", "split past 8, rest", (399, 1726, 32720, 32768, 32768, 0, 0, ASKED)),
    ("wide 256x256", "split, rest", (1986, 1334, 12688, 12800, 12800, 0, 0, ASKED)),
    ("wide 256x256", "whole", (389, 22049, 256, 256, 256, 0, 0, ASKED)),
    ("wide 256x256", "whole, rest", (406, 21933, 176, 272, 256, 112, 80, ASKED)),
]


def host_program(folder):
    """The host program that answers for the rule; None without a compiler."""
    hipcc = shutil.which("hipcc")
    if not hipcc:
        return None
    exe = os.path.join(str(folder), "q8_plan_check")
    cmd = [hipcc, "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2503_17707_amd", "q8"),
           os.path.join(HERE, "q8_plan_check.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


def plans(exe, rows):
    """[shape, splits, tail, full, kt, phases, skewed, bytes] of each [M, N, K, ldx, ldw, x, w, room]."""
    text = "\n".join(" ".join(map(str, r)) for r in np.asarray(rows).tolist())
    r = subprocess.run([exe], input=text + "\n", capture_output=True, text=True, timeout=120)
    assert r.returncode == 0
    out = np.array(r.stdout.split(), dtype=np.int64).reshape(-1, 8)
    assert len(out) == len(rows)
    return out


def label(K, plan):
    """What a launch is, in words."""
    shape, splits, tail, full, kt, phases, skewed, _ = (int(v) for v in plan)
    name, step, forms = KERNELS[shape]
    how = "whole" if splits == 1 else "split" if full == 0 else "last round split"
    return (name, how + (" past 8" if splits > 8 else "") + (", starts apart" if phases > 1 else "")
            + (", off lines" if forms and skewed else "") + (", rest" if K % step else ""))


def _spread(rng, n, lo, hi):
    return np.minimum(hi, np.exp(rng.uniform(np.log(lo), np.log(np.asarray(hi) + 0.999), n))).astype(np.int64).clip(min=lo)


def sample(seed, n):
    """n products: sizes over their range, many of K on whole steps and pages of 4 KB; rows packed, on lines and off them; no
    workspace, a large one, and any."""
    rng = np.random.default_rng(seed)
    pick = lambda *a: np.choose(rng.integers(0, len(a), n), a)  # noqa: E731
    M = pick(_spread(rng, n, 1, 64), _spread(rng, n, 1, 600), _spread(rng, n, 1, 8192))
    N = pick(_spread(rng, n, 1, 60000), 128 * _spread(rng, n, 1, 400))
    K = pick(16 * _spread(rng, n, 1, 2304), 128 * _spread(rng, n, 1, 288), 4096 * rng.integers(1, 10, n), 16 * _spread(rng, n, 1, 8191))
    line = (K + 127) // 128 * 128
    strides = rng.integers(0, 3, n)
    off = lambda: np.where(strides == 2, 16 * rng.integers(0, 8, n), 0)  # noqa: E731
    ld = lambda: np.where(strides == 0, K, line + off())  # noqa: E731
    room = pick(np.zeros(n, np.int64), np.full(n, ASKED), _spread(rng, n, 16, ASKED))
    return np.stack([M, N, K, ld(), ld(), (1 << 30) + off(), (1 << 30) + off(), room], 1)
