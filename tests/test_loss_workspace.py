"""A losses' workspace serves every smaller call too: its size never falls as
rows, vocabulary or pairs grow.  (Host only.)"""
import ctypes
import itertools

from paper_1802_08021_amd import sparcml as S


def size(op, pairs, rows, vocab):
    n = ctypes.c_size_t(0)
    assert S.lib().sparcml_workspace_size(op, pairs, rows, vocab, 1.0, ctypes.byref(n)) == S.OK
    return n.value


ROWS = sorted(set(range(1, 70)) | {r + d for r in (127, 170, 204, 255, 341, 511, 600, 1023, 1024, 4096, 2**20) for d in (0, 1, 2)}
              | {2**31 - 1})
VOCABS = [1, 7, 2048, 16383, 16384, 16388, 32767, 32768, 32776, 40000, 50001, 131072, 160000, 300000, 2**22, 2**31 - 1]


def test_sizes_never_fall():
    for op, pairs in itertools.chain(((S.OP_LOGPROB, 1), (S.OP_POLICY, 1)), ((S.OP_PREFERENCE, p) for p in (1, 4, 33, 65535))):
        table = [[size(op, pairs, r, v) for v in VOCABS] for r in ROWS]
        for r, row in enumerate(table):
            for v, n in enumerate(row):
                assert r == 0 or n >= table[r - 1][v], (op, pairs, ROWS[r], VOCABS[v])
                assert v == 0 or n >= row[v - 1], (op, pairs, ROWS[r], VOCABS[v])
    for rows, vocab in itertools.product(ROWS, VOCABS):
        sizes = [size(S.OP_PREFERENCE, p, rows, vocab) for p in (1, 2, 31, 32, 33, 400, 65535)]
        assert sizes == sorted(sizes)


def test_log_probabilities_need_no_place_for_a_loss_terms():
    """A row's (maximum, sum) and its token's logit: 12 bytes, and what the
    arrays' alignment takes."""
    for rows in (2**12, 2**20, 2**31 - 1):
        assert size(S.OP_LOGPROB, 1, rows, 131072) <= 12 * rows + 4096
