"""Limits that the header states, on the host: nothing is launched, no GPU is needed."""
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2510_11168_amd import build
    if not build.is_built():
        build.build()
    from paper_2510_11168_amd import binding
    return binding


def test_int8_products_have_a_tile_up_to_the_stated_sizes(b):
    sizes = [1, 2, 16, 17, 33, 64, 65, 128, 256, 257, 1000, 4096, 1 << 20, (1 << 27) - 16, (1 << 27) - 15, (1 << 29) + 1, (1 << 30) - 1, 1 << 30]
    seen = set()
    for M in sizes:
        for N in sizes:
            for K in (0, 1, 768, 2048, 131071):
                if -(-M // 256) * -(-N // 256) < 1 << 23:
                    t = b.elmo_int8_matmul_tile(M, N, K)
                    seen.add(t)
                    if t:                                        # what a launch takes: fewer than 2^32 work-items, 256 of a small tile, 512 of the others
                        assert -(-M // t) * -(-N // t) * (256 if t == 64 else 512) < 1 << 32
                    else:
                        assert M <= 32 and -(-N // 16) * 512 < 1 << 32
                else:
                    with pytest.raises(b.ElmoError):
                        b.elmo_int8_matmul_tile(M, N, K)
    assert seen == {0, 64, 128, 256}
    for M, N, K in ((0, 4, 4), (4, 0, 4), (4, 4, -1), (4, 4, 131072), ((1 << 30) + 1, 1, 1), (1, (1 << 30) + 1, 1)):
        with pytest.raises(b.ElmoError):
            b.elmo_int8_matmul_tile(M, N, K)


def test_int8_tiles_of_known_sizes(b):
    for M, N, K, tile in ((1, 4096, 4096, 0), (16, 8192, 8192, 0), (16, 131072, 768, 64), (32, 4096, 4096, 0), (33, 4096, 4096, 64), (37, 32003, 4096, 64), (512, 4096, 4096, 64),
                          (2048, 4096, 4096, 128), (8192, 14336, 4096, 256)):
        assert b.elmo_int8_matmul_tile(M, N, K) == tile, (M, N, K)


def test_more_rows_than_a_launch_takes_are_refused(b):
    """At the first number that the header excludes.  The addresses are never read: every call ends in the host's checks."""
    P = 4096
    norm = lambda rows, d: b._lib.elmo_rms_norm(P, d, b.ELMO_BF16, rows, d, None, 0, None, 0, 1e-6, None, 0, P, d, b.ELMO_BF16, None, None)  # noqa: E731
    assert norm(1 << 24, 2048) == -1 and norm(1 << 24, 8192) == -1 and norm(1 << 22, 8193) == -1 and norm(1 << 22, 16384) == -1
    assert norm((1 << 26) - 3, 1024) == -1 and norm((1 << 26) - 3, 1) == -1
    assert b._lib.elmo_sample(P, 8, b.ELMO_BF16, 1 << 22, 8, P, None, None, None, None, P, None, None, 0, None) == -1
    assert b._lib.elmo_distill(P, 8, b.ELMO_BF16, 1 << 23, 8, P, P, b.ELMO_FP32, 1, 1.0, None, P, None, 0, None, 0, None) == -1
    assert "launch" in b.elmo_last_error()
