"""Suffix calls over bf16 pages by the way that their launch takes: (query heads, kv heads, head_dim, requests, new tokens
each, greatest context).  test_page_dispatch_host.py holds the launch plan to it, test_gpu_page_rounding.py what each
way rounds."""
FEW = [   # at most 32 rows per kv head, keys split over a workgroup's waves
    (32, 8, 128, 1, 1, 1900), (32, 8, 128, 6, 3, 700), (28, 4, 128, 24, 4, 2600), (16, 1, 64, 80, 2, 1500), (8, 8, 64, 16, 13, 2000),
    (32, 8, 64, 16, 8, 4000), (32, 8, 128, 16, 8, 5000), (4, 4, 128, 64, 32, 1500), (5, 1, 64, 90, 3, 1000), (32, 8, 128, 30, 8, 2100)]
WHOLE = [(32, 8, 128, 12, 128, 190), (8, 2, 64, 16, 256, 1200), (32, 8, 64, 16, 128, 2000), (28, 4, 128, 20, 64, 3000)]
F32_SHARES = [(32, 8, 128, 8, 128, 6000), (28, 4, 128, 16, 64, 8000), (32, 8, 64, 16, 64, 4000)]
HALF_SHARES = [(32, 8, 128, 2, 40, 9001), (8, 2, 64, 2, 67, 4161), (28, 4, 128, 1, 128, 5000), (32, 8, 128, 1, 256, 1000),
               (32, 8, 128, 5, 40, 900)]
