"""What the losses over the vocabulary may take for their workspaces, as their header counts it: host arithmetic."""
import ctypes as C

from paper_2401_09135_b200 import binding as B
from test_ops_host_decoder import vocab_desc

MIB = 1 << 20


def taken(backward, **kw):
    n = C.c_uint64()
    assert B.lib().alsgd_vocab_bytes(vocab_desc(**kw), backward, C.byref(n)) == B.OK
    return n.value


def test_a_piece_of_dz_is_no_larger_than_said():
    """Narrow rows and no teacher: dz is nearly all there is.  A piece of 17 tiles' worth, rounded up to pairs of tiles, took 18."""
    for tiles in range(16, 80):
        assert taken(1, rows=30720, vocab=256 * tiles, dim=8) <= (256 + 8) * MIB, tiles
