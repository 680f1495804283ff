"""Scratch made for a batch serves every smaller one: sequences finish, and a program keeps what it made for the largest batch."""
import ctypes as C

import pytest

from paper_2303_06865_amd import binding as B


@pytest.mark.parametrize("vocab", [1, 2000, 8192, 8193, 50272, 256000])
@pytest.mark.parametrize("beams,n_best", [(1, 1), (4, 8), (3, 32), (16, 16)])
def test_select_workspace_of_a_batch_serves_smaller_ones(vocab, beams, n_best):
    L, cfg = B.lib(), B.fg_model_cfg(64, 1, 64, vocab, 64, 1e-5)
    size = lambda n, k, best: L.fg_beam_select_workspace_bytes(C.byref(cfg), n, k, best)  # noqa: E731
    sizes = [size(n, beams, n_best) for n in range(1, 600)]
    assert all(a > 0 and a <= b for a, b in zip(sizes, sizes[1:]))
    for n in (1, 2, 7, 18, 19, 80, 500):
        for k in range(1, beams + 1):
            for best in range(1, n_best + 1):
                assert size(n, k, best) <= size(n, beams, n_best), (n, k, best)


@pytest.mark.parametrize("nh,nkv,dh", [(32, 32, 128), (32, 8, 128), (12, 12, 64), (1, 1, 64), (34, 2, 64)])
@pytest.mark.parametrize("beams", [1, 2, 4, 5, 16])
def test_attention_workspace_of_a_batch_serves_smaller_ones(nh, nkv, dh, beams):
    L, cfg = B.lib(), B.fg_model_cfg(nh * dh, nh, 64, 64, 64, 1e-5)
    size = lambda groups, stride: L.fg_decode_attention_beams_workspace_bytes(C.byref(cfg), nkv, beams, groups * beams, stride)  # noqa: E731
    for stride in (1, 23, 24, 64, 100, 512, 5000):
        sizes = [size(n, stride) for n in range(1, 130)]
        assert all(a > 0 and a <= b for a, b in zip(sizes, sizes[1:])), stride
    for n in (1, 2, 3, 8, 64, 100):
        sizes = [size(n, stride) for stride in range(1, 700)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), n


def test_reorder_workspace_of_a_batch_serves_smaller_ones():
    size = B.lib().fg_beam_reorder_workspace_bytes
    for n in range(1, 200):
        assert all(0 < size(n, k) <= size(n, k + 1) for k in range(1, 16)) and size(n, 16) <= size(n + 1, 16)
