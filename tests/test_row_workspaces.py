"""Workspaces of sr_embed_grad and sr_add_norm_grad: enough for every size, no more than earlier builds asked for, and not many times what is used."""
import ctypes

import paper_2605_05802_amd as sr
from test_decoder_rows import row_plan  # noqa: F401  (a fixture)

NUMBERS = [*range(0, 140), 255, 256, 300, 511, 512, 513, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 4096, 8191, 8192, 8193, 16384, 49153, 50001, 65536, 100000, 262144, 2 ** 20 - 1, 2 ** 20]
WIDTHS = [*range(1, 20), 63, 64, 65, 255, 256, 257, 511, 512, 513, 1023, 1024, 1031, 2047, 2048, 3584, 4095, 4097, 8192, 16384, 18944, 70000, 1 << 18, (1 << 20) - 1, 1 << 20]


def test_partial_sums_of_tokens(row_plan):  # noqa: F811
    out = (ctypes.c_longlong * 8)()
    for width in WIDTHS:
        last = 0
        for n in NUMBERS:
            used = 0
            for single, bytes_ in ((0, 2), (1, 4)):
                row_plan.grad_plan(n, width, single, bytes_, out)
                end, room = out[6], out[7]
                assert end <= room == sr.embed_grad_workspace(n, width)
                used = max(used, end)
            assert room <= 65536 + 32 * n + (n // 8 + 64) * 4 * width        # a workspace that was enough stays enough
            assert room <= 4 * used + 65536 + 256 * width
            assert room >= last                                              # one for the largest list does for all
            last = room
    for n in NUMBERS:
        rooms = [sr.embed_grad_workspace(n, width) for width in WIDTHS]
        assert rooms == sorted(rooms)


def test_partial_sums_of_a_gain(row_plan):  # noqa: F811
    for rows in (0, 1, 2, 511, 512, 513, 1000, 2047, 2048, 2049, 10 ** 6, 2 ** 31 - 1):
        last = 0
        for width in range(1, 16385, 1 if rows in (513, 2048, 2 ** 31 - 1) else 61):
            used = max(4 * width * row_plan.norm_parts(rows, width, single) for single in (0, 1))
            room = row_plan.norm_workspace(rows, width)
            assert used <= room == sr.norm_grad_workspace(rows, width) <= min(rows, 2048) * 4 * width + 256
            assert room >= last and (width <= 512 or room <= 2 * used + 256)
            last = room
    assert all(sr.norm_grad_workspace(r, 3584) <= sr.norm_grad_workspace(r + 1, 3584) for r in range(3000))
