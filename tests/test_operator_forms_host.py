"""Which forms of the operators around a projection a batch takes, by the launches that the library's host side makes.  No device."""
import pytest

from tests.operator_forms import DEEP, TOKENS, WIDE_BACKWARD, WIDE_FORWARD
from tests.test_operators_host import run  # noqa: F401  (a fixture)


def of(names, threads, what):
    (n,) = [t for name, t in zip(names, threads) if what in name]
    return n


def test_wide_batches_have_several_pieces_in_a_workgroup(run):  # noqa: F811
    """256 threads for every tile and run of pieces, fewer than for every tile and piece (and in the backward 256 for every share of the sums beside them)."""
    fwd, bwd = [(c, "fwd", 1) for c in WIDE_FORWARD], [(c, "bwd", x) for c in WIDE_BACKWARD for x in (0, 1)]
    got = run([(name, (N, K, R, slots, x, M), -1) for (M, K, N, R, slots), name, x in fwd + bwd])
    for ((M, K, N, R, slots), name, _), (st, names, threads) in zip(fwd + bwd, got):
        groups = of(names, threads, "adapter_expandI" if name == "fwd" else "adapter_bwd_last") / 256
        if name == "bwd":
            groups -= slots * min(2048, (R * (N + K) // 4 + 255) // 256)
        tiles, pieces = M // 64 + slots + 1, ((N if name == "fwd" else K) + 127) // 128
        assert st == 0 and groups % tiles == 0 and groups / tiles <= (pieces + 1) // 2, (names, groups, tiles, pieces)


def test_deep_products_keep_four_pieces_ahead(run):  # noqa: F811
    """The forms with few enough registers a piece (16 rows, up to 32 of the rank), over more than the 32 pieces that are asked for at first."""
    for M, depth, R, slots in DEEP:
        assert depth // 64 > 32
        (st, names, _), = run([("fwd", (128, depth, R, slots, 1, M), -1)])
        assert st == 0 and any("adapter_shrinkILb0ELb0ELi1E" in n for n in names), names


@pytest.mark.parametrize("M,Hq,Hk,D,pairs,rows", TOKENS)
def test_large_batches_have_several_tokens_in_a_workgroup(run, M, Hq, Hk, D, pairs, rows):  # noqa: F811
    jobs = [(name, (Hq, Hk, D, pairs, pairing, 1, dtype, M), -1) for name in ("qk", "qk_bwd") for pairing in (0, 1) for dtype in (0, 1)]
    for st, names, threads in run(jobs):
        assert st == 0 and of(names, threads, "_kernel") / 256 <= (M + 1) // 2
