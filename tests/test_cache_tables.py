"""Tables far wider than the sequences, as a server allocates them for its longest request: the choice of kernel goes by the table's columns, the result does not."""
import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R
from tests.test_cache_attention import _attention_case, _check_attention, _gen, _say, workspace  # noqa: F401  (a fixture)

# (key heads, query heads per key head, d, block, T, lens, count, kernel over 3000 columns; z13: the 18 tiles of the fourth have 8 partial results of 16 896 bytes each, 13 times in 2^25 bytes)
CALLS = [
    (2, 4, 64, 64, 1, [777, 1, 0, 300], None, "rows16/z32"), (2, 3, 128, 16, 20, [300, 20, 65], [20, 20, 7], "rows32/z43"),
    (4, 4, 64, 64, 130, [130], None, "rows256/z21"), (2, 8, 128, 64, 70, [300, 70, 0], [70, 33, 0], "rows256/z13"), (2, 5, 64, 32, 110, [1000, 111], None, "rows256/z21"),
]


def _kernel(heads, group, d, bt, T, lens, columns=3000):
    return B.tir_debug_cache_kernel(len(lens), T, heads * group, heads, d, bt, columns)


def test_the_calls_take_the_kernels_that_wide_tables_choose():
    for heads, group, d, bt, T, lens, _, kernel in CALLS:
        assert _kernel(heads, group, d, bt, T, lens) == kernel, (T, _kernel(heads, group, d, bt, T, lens))


@pytest.mark.gpu
@pytest.mark.parametrize("cache,dtype", [("i8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("call", CALLS)
def test_short_sequences_in_wide_tables(workspace, call, cache, dtype):  # noqa: F811
    """What stands in the columns behind a sequence is no block, any block, or another sequence's."""
    import torch
    heads, group, d, bt, T, lens, count, kernel = call
    pool, table, q = _attention_case(_gen(T + d), cache, dtype, len(lens), T, heads, group, d, bt, lens)
    rest = torch.tensor([-1, 0, 2 ** 31 - 1, 1, pool[0].shape[0]], dtype=torch.int32).repeat(600)[:3000 - table.shape[1]]
    wide = torch.cat((table, rest.expand(len(lens), -1)), 1).contiguous()
    what = f"{T} tokens over {lens} in a table of {wide.shape[1]} columns, {kernel}"
    _say(what)
    _check_attention(pool, wide, q, lens, count, d ** -0.5, dtype, dtype, what)
