"""Products by the form that the library gives them (format of x, rows, h, h_out), each with a ragged K, past several turns of
its kernel's ring and of its scales: what test_gpu_mx_forms.py runs and test_mx_forms_cpu.py holds the choice of."""
from typing import NamedTuple

E4M3, E2M1 = 0, 1


class Form(NamedTuple):
    fmt: int
    rows: int
    h: int
    h_out: int
    kernel: str            # "stream NRxTG" (groups of 16 rows of W and of x) or "tile TNxTT" (columns and rows of y)
    ranges: int            # of K
    turned: bool = False   # one row of tiles, whose workgroups begin K at different places

    @property
    def name(self):
        fmt = "e4m3" if self.fmt == E4M3 else "e2m1"
        return f"{fmt}-{self.rows}x{self.h}x{self.h_out}-{self.kernel.replace(' ', '')}-{self.ranges}{'-turned' if self.turned else ''}"


def _both(rows, h, h_out, kernel, ranges=1, turned=False):
    return [Form(fmt, rows, h, h_out, kernel, ranges, turned) for fmt in (E4M3, E2M1)]


FORMS = [
    *_both(3, 5160, 136, "stream 1x1"),
    *_both(16, 5160, 4136, "stream 2x1"),
    *_both(4, 5160, 8200, "stream 2x1"),
    *_both(9, 5160, 8200, "stream 4x1"),
    *_both(20, 5160, 136, "stream 1x2"),
    *_both(31, 5160, 4136, "stream 2x2"),
    *_both(24, 5160, 8200, "stream 4x2"),
    *_both(72, 1064, 136, "tile 64x64"),
    *_both(64, 1992, 4104, "tile 64x64", 1, True),
    *_both(100, 8232, 264, "tile 64x64", 6),
    *_both(40, 4136, 1032, "tile 64x64", 5, True),
    *_both(72, 1064, 16392, "tile 128x64"),
    *_both(40, 1992, 28680, "tile 128x64", 1, True),
    *_both(136, 8232, 2056, "tile 128x64", 6),
    *_both(40, 8232, 4104, "tile 128x64", 6, True),
    *_both(200, 1064, 16392, "tile 128x128"),
    *_both(72, 1992, 28680, "tile 128x128", 1, True),
    Form(E4M3, 200, 8232, 4104, "tile 128x128", 6),
    Form(E2M1, 200, 8232, 2056, "tile 128x128", 6),
    *_both(72, 16424, 4104, "tile 128x128", 7, True),
    *_both(264, 1064, 28680, "tile 256x256"),
    *_both(2056, 1064, 4104, "tile 256x256"),
    *_both(200, 1992, 57352, "tile 256x256", 1, True),
    *_both(512, 16424, 4104, "tile 256x256", 7),
    *_both(136, 16424, 8200, "tile 256x256", 7, True),
    *_both(136, 8232, 28680, "tile 256x256", 2, True),
]
