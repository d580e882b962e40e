"""Sizes at which the kernels of the products in 8 bits reach their steady state: stages that are filled again while others are
multiplied, and scales of W of a second run of 64 blocks.  (M, N, K); test_host_fp8_plan.py asks which kernel each takes."""

# more than 64 blocks of 128
LONG = [(9, 64, 8459), (250, 513, 8449), (500, 513, 8303), (700, 1500, 8459), (777, 700, 8303), (1500, 1500, 8303), (1300, 3001, 8449),
        (2000, 2000, 8300), (2500, 3000, 8449), (3000, 3000, 8500), (2500, 5000, 8333)]
# a few more than the stages hold
SHORT = [(700, 1500, 603), (1500, 8200, 600), (4096, 4096, 1000), (1300, 5000, 777), (8000, 1000, 770), (777, 4096, 650), (1300, 6000, 681),
         (2500, 1500, 1000), (2000, 2000, 1111), (520, 700, 1031)]
