"""Sizes at which the kernels of the experts' products are to reach their steady state: more blocks of the reduction than their stages hold, and more than 64.
(tokens, picks, experts, outputs, inputs)."""

SIZES = [(30, 2, 4, 300, 1300), (250, 2, 8, 1500, 1000), (1000, 2, 4, 2048, 900), (3000, 2, 8, 2048, 1111), (4096, 2, 8, 4096, 1000), (2500, 4, 8, 3000, 700),
         (600, 2, 4, 4096, 1000), (64, 2, 8, 4096, 4096), (200, 1, 2, 513, 8449), (2, 2, 4, 64, 8459), (900, 2, 4, 700, 8303), (2000, 2, 4, 2000, 8300),
         (300, 2, 2, 4096, 8300), (100, 2, 2, 1500, 8300), (1500, 1, 16, 1500, 1200), (2000, 1, 2, 3000, 8449)]
