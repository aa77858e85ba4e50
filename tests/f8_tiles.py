"""Products that between them run every kernel of the 8-bit product on sizes that
end inside a tile, over several words of scales, with rows of c on and off the
alignment of wide stores: (m, n, k, output, kernel, workgroups that share k, rows
of c in a wider array). The kernel of each is what the host check of the plans
(test_plans_host.py) finds; the GPU test (test_gpu_f8_tiles.py) runs them."""

PRODUCTS = [
    (1237, 8191, 1300, "bf16", "256x256", 1, False),
    (1237, 8192, 1300, "bf16", "256x256", 1, True),
    (2311, 4096, 2050, "bf16", "256x256", 1, False),
    (3000, 5000, 900, "bf16", "256x256", 1, False),
    (2001, 2103, 1200, "f32", "128x128", 1, False),
    (2001, 2104, 1300, "f32", "128x128", 1, False),
    (2001, 2104, 2050, "f32", "128x128", 1, True),
    (2001, 2103, 1200, "bf16", "128x128", 1, False),
    (2001, 2104, 1300, "bf16", "128x128", 1, False),
    (700, 1001, 1300, "f32", "64x64", 1, False),
    (300, 203, 5000, "bf16", "64x64", 2, False),
    (300, 204, 5000, "f32", "64x64", 2, True),
    (50, 303, 5000, "bf16", "thin", 5, False),
    (17, 20003, 1300, "f32", "thin", 1, False),
    (3, 304, 9000, "bf16", "thin", 8, True),
]
