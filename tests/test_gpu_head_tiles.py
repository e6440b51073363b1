"""The head in every tile and form of its products, at odd remainders: which one a size takes is a rule on rows, width, vocabulary and type,
and the sizes here were picked so that each comes up, for one target and for a teacher's entries.

    tiles of 256 in all four products, several pieces of the vocabulary (a teacher's entries come off afterwards)   the first two
    tiles of 128, dx in shares of the vocabulary (a teacher's entries come off in the tile)                         the next two
    few rows: tiles of 256 and of 128 with three planes of d, the wide tile of dx                                   the next three
    few rows, several pieces: rows through LDS, straight from memory, float32                                       the last three"""
import pytest

from .test_gpu_head_ranges import _case, _check
from .test_gpu_training import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [0, 20])
@pytest.mark.parametrize("dtype,rows,hidden,vocab", [(BF16, 4100, 1544, 45003), (F32, 2049, 1032, 70001),
                                                     (BF16, 700, 520, 3001), (F32, 520, 264, 9001),
                                                     (BF16, 150, 264, 40003), (BF16, 150, 1032, 20003), (BF16, 40, 2056, 20003),
                                                     (BF16, 150, 8, 600001), (BF16, 150, 9, 600001), (F32, 150, 8, 600001)])
def test_every_tile(dtype, rows, hidden, vocab, top):
    _check(f"{rows}x{hidden}x{vocab} top {top} {dtype}", _case(rows, hidden, vocab, dtype, top, seed=hidden), 2.0 if top else 1.0)
