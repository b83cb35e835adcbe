"""What the GPU tests of the distillation's rows allow is less than one entry of the longest of them is worth."""
import numpy as np

import test_gpu_distill_rows as rows


def test_one_of_equal_entries_is_seen():
    n = float(max(rows.LENGTHS))
    for wrong in (n - 1, n + 1):
        for u, soft, hard in ((1.0, 1.0, 0.0), (2.0, 0.5, 0.25), (4.0, 0.0, 1.0)):
            want = (soft * u * u + hard) * np.log(n)
            assert abs((soft * u * u + hard) * np.log(wrong) - want) > want * 6 * 2.0 ** -24
            assert abs(1 / wrong - 1 / n) > 8 * 2.0 ** -24 / n          # (each entry of a gradient in fp32)


def test_the_largest_of_a_row_is_seen():
    rng = np.random.default_rng(0)
    for V in rows.LENGTHS[2:]:
        for pieces, step in ((8, False), (8, True), (4, False), (4, True)):
            n, turn = rows.threads(V, pieces, step)
            z = rng.standard_normal(V)
            rel = 2 * (8 * 50 + V / n + 64) * 2.0 ** -24
            for u in (1.0, 2.0):
                rest, one = np.exp(z / u).sum(), np.exp(40 / u)
                want = np.log(rest + one)
                for wrong in (np.log(rest), np.log(rest + 2 * one)):
                    assert abs(wrong - want) > 0.5 > 4 * (3 * rel + 50 * 2.0 ** -22)
            head = 3
            at = rows.edges(V, head, pieces, n, turn)
            assert {0, V - 1, head} <= set(at) and (V - head) // pieces * pieces + head - 1 in at


def test_every_way_through_a_row_is_taken():
    for pieces in (8, 4):
        for step in (False, True):
            taken = {rows.threads(V, pieces, step) for V in rows.LENGTHS}
            ways = {(64, 64), (256, 256), (1024, 4096)} | ({(512, 512), (1024, 1024)} if step else {(256, 1024), (512, 2048)})
            assert taken == ways, (pieces, step, ways - taken)
