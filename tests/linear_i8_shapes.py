"""8-bit products (rows, outputs, inputs) by the kernel that each is planned by on 256 CUs, in both types, with a residual and
without: first aligned rows of whole 16-byte chunks, then others."""

KERNELS = ("tile256", "tile128", "tile64", "deep128", "deep64", "staged128", "staged64", "staged32", "split16x16", "split32x16", "split64x16", "split32x32", "split64x32",
           "split32x64", "split64x64", "short")
DIRECT = {"tile256": [(8000, 4080, 64)], "tile128": [(8000, 2297, 16)], "tile64": [(700, 1000, 16)], "deep128": [(4090, 809, 4608)], "deep64": [(1025, 1000, 4096)],
          "split16x16": [(24, 1040, 1024)], "split32x16": [(17, 2297, 512)], "split64x16": [(300, 816, 4608), (297, 809, 1920)], "split32x32": [(297, 512, 4096)],
          "split64x32": [(97, 2297, 1920)], "split32x64": [(200, 2304, 4608), (203, 2297, 1920)], "split64x64": [(500, 1040, 4096)]}
OTHERS = {"staged128": [(3000, 2297, 61)], "staged64": [(700, 4080, 61)], "staged32": [(1025, 809, 61)], "split16x16": [(31, 2040, 261)], "split32x32": [(17, 2297, 645)],
          "split64x64": [(97, 2297, 4093)], "short": [(297, 512, 13)]}
SHAPES = [(kernel, shape) for table in (DIRECT, OTHERS) for kernel, shapes in table.items() for shape in shapes]
