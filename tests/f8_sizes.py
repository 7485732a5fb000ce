"""Sizes of 8-bit floating-point products and gated blocks by the form of the kernels that they lead to: (tiles, in K ranges) -> (m, n, k).  The
forms are checked on the CPU, the results on the GPU."""
THIN, SMALL, MIDDLE, LARGE = range(4)

PRODUCTS = {
    (THIN, False): [(33, 130, 1111)],
    (SMALL, False): [(257, 20001, 500), (129, 127, 255)],
    (SMALL, True): [(300, 201, 5000)],
    (MIDDLE, False): [(2001, 1999, 1500)],
    (MIDDLE, True): [(257, 601, 16000)],
    (LARGE, False): [(257, 60001, 500)],
    (LARGE, True): [(1025, 1001, 20000)],
}
GATED = {
    (THIN, False): [(40, 101, 1111)],
    (SMALL, False): [(500, 201, 777), (1500, 1001, 385)],
    (SMALL, True): [(150, 131, 20000)],
    (MIDDLE, False): [(500, 4001, 1000)],
    (MIDDLE, True): [(257, 301, 16000)],
    (LARGE, False): [(2901, 1501, 500)],
    (LARGE, True): [(1025, 1001, 10000)],
}
