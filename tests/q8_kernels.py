"""Decoding cases over the 8-bit cache and the kernel that each is for (test infrastructure)."""
TC, MMA = True, False

# (B, n, Hq, Hkv, Dh, P, T, L): scores that climb, fall or jump on the tcgen05 kernel at head dim 64, whose O has 64 rows:
# 32, 48 and 64 query rows of a K/V head, groups of them, and few rows of many positions
CHANGE = [(2, 4, 16, 2, 64, 16, 16, 700), (3, 4, 48, 4, 64, 32, 8, 500), (2, 8, 16, 2, 64, 8, 2, 300), (2, 4, 96, 4, 64, 20, 5, 400),
          (90, 4, 4, 4, 64, 32, 1, 760)]
# (B, n, Hq, Hkv, Dh, P, T, L): one wave shared by uneven sequences there
WAVE = [(2, 4, 32, 4, 64, 32, 8, 16000)]
# (kernel, n, Hq, Hkv, Dh, P, T, L): queries far from 1, explicit scales
SIZES = [(TC, 2, 8, 2, 128, 8, 2, 80), (TC, 4, 12, 1, 256, 16, 4, 80), (TC, 4, 8, 1, 256, 16, 16, 80), (TC, 4, 12, 2, 64, 16, 16, 80),
         (MMA, 2, 8, 2, 128, 3, 1, 80), (MMA, 1, 8, 2, 64, 16, 16, 200), (MMA, 4, 24, 2, 256, 1, 1, 60), (MMA, 4, 12, 1, 128, 1, 1, 60)]
# (kernel, n, Hq, Hkv, Dh, P, T, L, window): pages given up behind the window, which starts inside a page, a tile, a piece
GIVEN_UP = [(k, n, Hq, Hkv, Dh, P, T, L, w) for k, n, Hq, Hkv, Dh, P, T, L in
            [(TC, 2, 16, 2, 128, 16, 16, 300), (TC, 4, 12, 1, 128, 20, 5, 200), (TC, 4, 24, 2, 256, 16, 4, 200), (TC, 4, 16, 2, 64, 32, 8, 200),
             (MMA, 2, 8, 2, 128, 3, 3, 200), (MMA, 1, 8, 2, 64, 16, 4, 400), (MMA, 4, 24, 2, 256, 1, 1, 150)] for w in (97, 131, 256, 300)]
