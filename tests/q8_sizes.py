"""Sizes (m, N, K) of d2c_q8_linear that reach each of its kernels, and the product's definition in elementary 64-bit operations of torch.

LINEAR: (kernel, row tiles, column tiles, whether the contraction is split) -> sizes.  None is a multiple of its tiles; N with and without whole
groups of four, one and several groups of rows, chunks of the contraction even and odd in number."""
import torch

SMALL, STREAM, TILE = 0, 1, 2
LINEAR = {
    (SMALL, 1, 1, False): [(1, 20, 8), (13, 6143, 1000), (15, 1002, 2040)],
    (STREAM, 1, 1, False): [(1, 20, 2120), (9, 6150, 520), (15, 3001, 2200)],
    (STREAM, 1, 1, True): [(1, 17, 4112), (11, 1030, 18936)],
    (STREAM, 1, 2, False): [(1, 8186, 8), (12, 8204, 264)],
    (STREAM, 2, 1, False): [(17, 17, 8), (31, 1000, 520)],
    (STREAM, 2, 1, True): [(17, 18, 4672), (29, 1036, 12280)],
    (STREAM, 2, 2, False): [(20, 8204, 264), (31, 8418, 1000)],
    (TILE, 1, 1, False): [(33, 20, 8), (34, 20, 520), (35, 17, 520), (147, 1131, 776)],
    (TILE, 1, 1, True): [(33, 20, 1840), (34, 17, 1808)],
    (TILE, 2, 1, False): [(130, 4098, 1016), (2166, 140, 520)],
    (TILE, 2, 1, True): [(681, 20, 2768), (674, 18, 2600)],
    (TILE, 3, 1, False): [(34, 16764, 528), (67, 10889, 528), (300, 4100, 1016)],
    (TILE, 3, 1, True): [(33, 2234, 5200), (1387, 20, 4104)],
    (TILE, 4, 1, False): [(49, 18668, 528), (102, 11126, 544)],
    (TILE, 4, 1, True): [(50, 2710, 9240), (1842, 20, 5240)],
    (TILE, 6, 1, False): [(142, 11112, 528), (139, 11013, 520)],
    (TILE, 6, 1, True): [(66, 2780, 12664), (2053, 17, 9976)],
    (TILE, 8, 1, False): [(99, 16868, 520), (193, 11094, 536)],
    (TILE, 8, 1, True): [(99, 5784, 10088), (2124, 17, 20080)],
    (TILE, 4, 2, False): [(143, 16840, 520), (129, 18343, 520)],
    (TILE, 4, 2, True): [(33, 16604, 8336), (1329, 134, 39520)],
    (TILE, 6, 2, False): [(141, 22948, 552), (129, 22850, 536)],
    (TILE, 6, 2, True): [(65, 16395, 8360), (2099, 152, 28072)],
    (TILE, 8, 2, False): [(213, 21900, 520), (195, 21858, 536)],
    (TILE, 8, 2, True): [(100, 16924, 8864), (98, 17174, 9200)],
    (TILE, 8, 3, False): [(321, 21992, 520), (193, 34817, 520)],
    (TILE, 8, 3, True): [(100, 33494, 8480), (132, 11196, 37800)],
}


def linear(a, w):
    """As q8_reference.linear, on the tensors' own device: sizes of billions of products."""
    def rows(x):
        x = x.double()
        bad = ~torch.isfinite(x).all(1)
        x = torch.where(bad[:, None], 0.0, x)
        amax = x.abs().amax(1)
        s = torch.where(amax < 2.0 ** -100, 0.0, (amax / torch.full_like(amax, 127)).float().double())
        c = torch.where(s[:, None] == 0, 0.0, torch.round(x / torch.where(s == 0, 1.0, s)[:, None]))
        return c.clamp_(-127, 127), torch.where(bad, float("nan"), s).float()

    (qa, sa), (qw, sw) = rows(a), rows(w)
    return torch.matmul(qa, qw.t().contiguous()).float() * sa[:, None] * sw, sw
