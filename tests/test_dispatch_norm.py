"""The rules that pick layer norm's forward kernels (csrc/dispatch.hpp), on the host, against measured times."""
import collections

from tests import dispatch_host as H

# with dropout and sum, rows, columns | us of the forward in the variant of that width with 8, 7, 6, 5, 4 waves on a SIMD where a lane has one chunk of a row (1025 to 2048 columns),
# with 7, 6, 5, 4 where it has two, with 4, 3, 2 where it has two and adds dropout and sum.  bf16, the last twelve fp32
TIMES = """
0 131072 4096 | 399.6 401.5 383 410.1; 0 16384 4096 | 50.52 49.03 48.51 52.27; 0 30000 3000 | 66.7 67.83 72.5 82.68
0 8192 5001 | 34.67 34.72 41.21 42.24; 0 32768 8192 | 189.4 183.5 196.2 195.4; 0 16000 5120 | 64.22 64.38 79.53 79.65
0 20000 900 | 14.69 14.45 15.13 15.76; 0 131072 1024 | 97.24 96.59 94.07 100.1; 0 100000 128 | 9.98 10.35 10.2 10.33
0 500000 256 | 90.46 91.25 90.15 95.4; 0 16384 2048 | 22.34 22.19 22.55 22.2 23.64; 0 131072 2048 | 194.1 195.9 199.4 196 199.4
0 20000 1500 | 23.11 24 24.92 26.22 29.9; 1 131072 4096 | 823.4 802.8 881.3; 1 16384 4096 | 93.71 95.06 115.2
1 30000 3000 | 139.4 153.5 201.1; 1 8192 5001 | 93.8 133 134; 1 32768 8192 | 377 447.6 446.9
1 16000 5120 | 128.4 183.4 185.2; 1 20000 900 | 30.32 32.18 35.31; 1 131072 1024 | 193.3 191 224.9
1 100000 128 | 19.26 20.53 23.56; 1 500000 256 | 178 195.1 250.2; 1 16384 2048 | 48.36 48.54 48 48.06 51.69
1 131072 2048 | 388.3 396.4 402.6 396 406.1; 1 20000 1500 | 54.88 58.2 63.48 69.04 78.55; 0 65536 4096 | 402.1 402.3 401.7 399.7
0 8192 5001 | 67.21 67.48 64.74 64.76; 0 16384 8192 | 199.2 199.2 195.6 196; 0 65536 2048 | 208.1 209.3 209.8 210.8 200.4
0 3001 1111 | 6.9 7.06 7.08 7.17 7.49; 0 20000 900 | 32.85 32.83 32.67 32.45; 1 65536 4096 | 809.9 805.5 820.5
1 8192 5001 | 129.1 125.1 125.2; 1 16384 8192 | 398.9 399.2 407.4; 1 65536 2048 | 414.7 415.6 416.3 414.8 412.5
1 3001 1111 | 11.1 10.93 11.27 11.32 11.79; 1 20000 900 | 61.31 61.27 60.36
"""
LANES = "(norm_rows(E) == NormRows::k16x2 ? 16 : norm_rows(E) == NormRows::k64x2 ? 64 : norm_rows(E) == NormRows::k512x2 ? 512 : norm_rows(E) == NormRows::k1024x2 ? 1024 : 256)"
CHUNKS = "(norm_rows(E) == NormRows::k256x1 ? 1 : 2)"


def test_limits_hold_the_row():
    widths = [1, 8, 255, 256, 257, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384]
    for E, (lanes, chunks, most) in zip(widths, H.ask([(E,) for E in widths], LANES, CHUNKS, "kNormMaxCols", names=("E",))):
        assert lanes * chunks * 8 >= E and most == 16384
    assert [r[:2] for r in H.ask([(E,) for E in widths[3:12]], LANES, CHUNKS, names=("E",))] == [(16, 2), (64, 2), (64, 2), (256, 1), (256, 1), (256, 2), (256, 2), (512, 2), (512, 2)]


def test_waves_against_their_times():
    """For each variant the chosen number costs, on average over its shapes, at most 1 % more than the best number does."""
    table = list(H.read_table(TIMES))
    asked = H.ask([shape for shape, _ in table], LANES, CHUNKS, f"norm_fwd_waves({LANES}, {CHUNKS}, S)", names=("S", "M", "E"))
    groups = collections.defaultdict(list)
    for (shape, us), (lanes, chunks, waves) in zip(table, asked):
        options = (8, 7, 6, 5, 4) if chunks == 1 else (4, 3, 2) if shape[0] else (7, 6, 5, 4)
        assert len(us) == len(options)
        groups[lanes, chunks, shape[0]].append((options.index(waves), [t / min(us) for t in us]))
    assert len(groups) == 10
    for variant, shapes in groups.items():
        mean = [sum(r[i] for _, r in shapes) / len(shapes) for i in range(len(shapes[0][1]))]
        assert mean[shapes[0][0]] <= 1.01 * min(mean), (variant, mean)
