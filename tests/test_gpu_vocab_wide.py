"""Losses over the vocabulary at wide rows, up to the widest that are taken."""
import pytest

from test_gpu_vocab import check
from vocab_ref import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("rows,vocab,dim", [(1, 300, 16384), (70, 700, 4104), (130, 1000, 16384), (600, 520, 8200), (2000, 3000, 4096)])
def test_wide_rows(rows, vocab, dim, top):
    check(Problem(rows, vocab, dim, top=top, seed=rows))
