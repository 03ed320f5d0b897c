"""What the losses over the vocabulary may take for their workspaces, as their header counts it: host arithmetic."""
import ctypes as C
import itertools

import pytest

from paper_2401_09135_b200 import binding as B
from test_ops_host_decoder import vocab_desc

MIB = 1 << 20


def taken(backward, **kw):
    n = C.c_uint64()
    assert B.lib().alsgd_vocab_bytes(vocab_desc(**kw), backward, C.byref(n)) == B.OK
    return n.value


def counted(backward, rows, vocab, dim, top):
    rows, tiles = -(-rows // 256) * 256, -(-vocab // 256)
    n = rows * (2 * dim + 32) + 16384
    if top:
        n += rows * (8 * top + 4 * (tiles + 1))
    if not backward:
        return n + rows * (8 * tiles + 4 * max(1, top))
    return n + max(256 * MIB, 8192 * rows) + max(256 * MIB, 4 * rows * dim) + 256 * MIB


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("top", [0, 1, 128])
def test_the_workspace_is_what_its_account_says(backward, top):
    for rows, vocab, dim in itertools.product([1, 77, 300, 8144, 30208, 65536, 70001, 1 << 20], [1, 5000, 8704, 32000, 100003, 1 << 20], [8, 384, 1024]):
        kw = dict(rows=rows, vocab=vocab, dim=dim, top=top)
        assert taken(backward, **kw) <= counted(backward, **kw), kw


def test_a_piece_of_dz_is_no_larger_than_said():
    """Narrow rows and no teacher: dz is nearly all there is.  A piece of 17 tiles' worth, rounded up to pairs of tiles, took 18."""
    for tiles in range(16, 80):
        assert taken(1, rows=30208, vocab=256 * tiles, dim=8) <= (256 + 8) * MIB, tiles
