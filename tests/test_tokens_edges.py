"""The token operators at the edges of their ranges, on the CPU."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CLANG = shutil.which("clang++", path="/opt/rocm/llvm/bin" + os.pathsep + os.environ["PATH"])


@pytest.fixture(scope="module")
def lib():
    from paper_1505_03851_amd import _lib
    return _lib.load()


# ---- the embedding's gradient of rows of up to 2^31 - 1 columns


@pytest.fixture(scope="module")
def grad_columns(tmp_path_factory):
    if CLANG is None:
        pytest.skip("no clang++")
    exe = str(tmp_path_factory.mktemp("columns") / "grad_columns")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-w",
                    "-I", os.path.join(HERE, "leaf_host"),
                    "-I", os.path.join(ROOT, "paper_1505_03851_amd", "csrc"),
                    os.path.join(HERE, "leaf_host", "grad_columns.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("D", [1, 2, 5, 7, 8, 63, 64, 65, 129, 257, 511, 512, 513, 1003, 2055,
                               2 ** 30 - 1, 2 ** 30, 2 ** 30 + 9, 2 ** 30 + 1000, 2 ** 31 - 513,
                               2 ** 31 - 512, 2 ** 31 - 511, 2 ** 31 - 8, 2 ** 31 - 1])
def test_columns_of_a_row(grad_columns, D):
    """Every column is written by one lane, and read at its own address."""
    run = subprocess.run([grad_columns, str(D)], stdout=subprocess.PIPE, text=True, timeout=60)
    assert run.returncode == 0, run.stdout


def test_runs_fit_a_launch(lib):
    """A wavefront's run of tokens grows with the columns, so that the launch holds
    its wavefronts (2^26): the parts of words that cross runs stay below 2^38 bytes
    and the workspace with them."""
    f = lib.lda_embed_grad_workspace_bytes
    for D in (2 ** 20, 2 ** 24, 2 ** 28 + 5, 2 ** 30, 2 ** 31 - 1):
        for N in (129, 5000, 1 << 20, 2 ** 31 - 1):
            assert f(N, 5, D) <= 2 ** 38 + 64 * N + 2 ** 20, (N, D)
    assert f(1 << 20, 32_768, 256) < 2 ** 25 + 64 * 2 ** 20  # the usual run: 256 tokens


# ---- sizes past 32 bits


def test_workspace_of_sizes_past_32_bits():
    """2^32 + a few is not a few: unsupported, as the header says of what is 0."""
    import paper_1505_03851_amd as lda
    many = 2 ** 32 + 40_000
    assert lda.embed_grad_workspace_bytes(1000, 40_000, 8) > 0
    assert lda.draw_logits_workspace_bytes(3, 40_000) > 0
    assert lda.embed_grad_workspace_bytes(1000, many, 8) == 0
    assert lda.embed_grad_workspace_bytes(1000, 8, many) == 0
    assert lda.draw_logits_workspace_bytes(3, many) == 0


# ---- one history for every row


def test_history_rows(lib):
    """A distance of 0 (one row for all) passes the checks, one below the capacity
    does not.  B = 0 returns after the checks of the rules."""
    import ctypes
    from paper_1505_03851_amd import _lib
    from paper_1505_03851_amd._tokens import LogitRules
    A, value = 4096, _lib.STATUS["LDA_ERR_VALUE"]
    for apart, want in ((0, 0), (5, 0), (9, 0), (4, value), (1, value), (-5, value)):
        r = ctypes.byref(LogitRules(A, apart, 5, A, None, None, None, None, None, 0, None, 0))
        assert lib.lda_penalise_logits(A, 40, A, 40, 0, 40, 0, r, None) == want, apart
        assert lib.lda_draw_logits(A, 40, 0, 40, 0, r, None, None, A, A, A, A, A, 1 << 20,
                                   None) == want, apart
