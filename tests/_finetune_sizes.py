"""Sizes at which the kernels of adapters and distillation go through their loops: workgroups that take several tiles, several
adapters, row after row.  tests/test_finetune_reach.py checks on the CPU that every kernel and every such loop is
reached, tests/test_gpu_finetune_loops.py compares the results with the definitions."""

# tokens, inp, out, rank, adapters, order of the tokens ("segments": requests one after the other; "mixed")
ADAPTERS = [
    (16384, 4096, 1024, 16, 4, "segments"), (17000, 1024, 4096, 8, 3, "mixed"), (16001, 2048, 4104, 12, 5, "segments"),
    (8192, 2048, 8192, 32, 8, "mixed"), (8200, 4104, 8192, 20, 7, "segments"), (4096, 8192, 8200, 64, 8, "segments"),
    (5000, 8200, 8192, 50, 6, "mixed"), (4096, 1024, 8192, 100, 5, "segments"), (6000, 4096, 8200, 128, 3, "mixed"),
    (3001, 8192, 4096, 90, 2, "mixed"), (2500, 2056, 4104, 96, 40, "mixed"), (9001, 8192, 4096, 32, 3, "segments"),
    (40000, 1000, 264, 16, 4, "mixed"), (30000, 264, 72, 9, 7, "mixed"), (26001, 264, 1024, 30, 5, "segments"), (26003, 1024, 504, 32, 3, "mixed"),
    (13000, 1024, 1024, 64, 4, "segments"), (13001, 512, 264, 100, 3, "mixed"), (30007, 264, 504, 48, 5, "segments"),
    (512, 8192, 264, 16, 1, "one"),
]
# ... and for few tokens, where a workgroup has one tile
ADAPTERS_FEW = [(64, 8192, 8192, 16, 32, "mixed"), (192, 8192, 520, 33, 3, "segments"), (130, 8192, 264, 64, 2, "mixed"),
                (192, 8192, 136, 128, 2, "mixed"), (192, 16384, 64, 10, 2, "mixed"), (96, 8192, 1032, 12, 5, "mixed"),
                (100, 1024, 264, 20, 3, "mixed"), (190, 4096, 72, 32, 4, "segments"), (192, 3000, 512, 64, 4, "mixed"),
                (185, 6000, 264, 32, 2, "segments")]

# tokens, words, entries of a list; half as many words in fp32
DISTILL = [
    (5000, 8191, 40), (12500, 8001, 20), (14001, 8191, 8),                  # 256 threads, 4 pieces each
    (4001, 10001, 33), (4500, 12001, 64), (7001, 16001, 10),                # 8
    (2300, 16501, 100), (2300, 30001, 17), (3301, 32001, 64),               # 16
    (1100, 33001, 64), (1101, 60001, 30), (1700, 65001, 12),                # 512 threads
    (601, 65601, 50), (600, 131071, 64), (801, 131072, 5),                  # 1024 threads
    (70, 140001, 30), (401, 151937, 64), (700, 151936, 9),                  # too long for registers
]
