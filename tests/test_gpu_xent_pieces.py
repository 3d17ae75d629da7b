"""Loss over a vocabulary that is taken in several pieces, and logits whose contraction is cut on every tile: sizes at which the number of
tokens that do have a class, which only the device knows, leaves several pieces or slices.  Bounds: see test_gpu_xent."""
import numpy as np
import pytest
import torch

import paper_2411_11038_amd as ef

from test_gpu_xent import check_all, make

pytestmark = pytest.mark.gpu


def up(n, m):
    return -(-n // m) * m


def pieces(T, D, V, dtype, direct, tokens, backward):
    """(number, classes of a whole one) of the pieces for so many tokens with a class: those whose G, or whose classes laid out anew,
    fit their limits of 2^26 to 2^28 and of 2^26 elements"""
    parts = 1 if dtype == "bf16" else 3
    most = up(V, 256)
    if not direct:
        most = min(most, max(2 ** 26 // (up(D, 64) * parts) // 256 * 256, 1024))
    if backward:
        elems = min(max(up(T, 256) * parts * up(up(V, 2) // 2, 256), 2 ** 26), 2 ** 28)
        most = min(most, max(elems // (up(max(tokens, 1), 256) * parts) // 256 * 256, 1024))
    size = up(-(-V // -(-V // most)), 256)
    return -(-V // size), size


def around(t, V, size):
    """the first and last classes of the pieces among the targets"""
    edges = [c for p in range(0, V, size) for c in (p, min(p + size, V) - 1)]
    t[: len(edges)] = edges
    return torch.from_numpy(t).cuda()


# classes as they lie (whole K stages, whole 16 bytes), and laid out anew
@pytest.mark.parametrize("D", [64, 72, 65])
def test_pieces_of_the_gradient(D):
    """bf16: dh adds the pieces up in fp32 and leaves as bf16 with the last one, which is ragged"""
    T, V = 4300, 16100
    h, w, t, hd, wd, _ = make(T, D, V, "bf16", D, ignored=0.02)
    n, size = pieces(T, D, V, "bf16", D % 8 == 0, int((t >= 0).sum()), True)
    assert n == 2 and V % size
    check_all(h, w, t, hd, wd, around(t, V, size), "bf16")


@pytest.mark.parametrize("T,D,V,dtype,number", [(40, 2050, 24001, "f32", 3), (300, 2050, 24001, "f32", 3), (40, 2050, 33001, "bf16", 2),
                                                (700, 2050, 33001, "bf16", 2)])
def test_pieces_of_classes_laid_out_anew(T, D, V, dtype, number):
    """forward and backward; tiles of 64, 128 and 256 classes, whose statistics lie behind those of the pieces before"""
    h, w, t, hd, wd, _ = make(T, D, V, dtype, T, ignored=0.1)
    tokens = int((t >= 0).sum())
    n, size = pieces(T, D, V, dtype, False, tokens, False)
    assert n == number and V % size and pieces(T, D, V, dtype, False, tokens, True)[0] >= number
    check_all(h, w, t, hd, wd, around(t, V, size), dtype)


# contraction of the logits cut: tiles of 256 (195 of them, one slice) and, with fewer tokens than the host knows of, 65 in three slices; of
# 128, 129 in three slices
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,ignored", [(600, 0.0), (600, 0.62), (100, 0.0)])
def test_slices_of_logits(T, ignored, dtype):
    check_all(*make(T, 3136, 16500, dtype, T, ignored=ignored), dtype)
