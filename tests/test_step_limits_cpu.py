"""Sizes at the cross entropy's documented limits."""
import pytest

from paper_2608_11034_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


@pytest.mark.parametrize("rows,vocab", [(1 << 24, 1 << 21), (1 << 21, 1 << 24), (5931641, 5931642)])
@pytest.mark.parametrize("dtype", [binding.DT_BF16, binding.DT_F16])
def test_rows_times_vocabulary(rows, vocab, dtype):
    assert rows * vocab <= 1 << 45
    forward, backward = binding.scout_loss_workspace(dtype, rows, 64, vocab)
    tiles = -(-rows // 256) * -(-vocab // 256)
    assert tiles < (1 << 31) - 1000 and forward >= rows * 64 * 2 + 8 * rows * (vocab // 128) and backward >= rows * 64 * 6
    for more in ((rows + 1, vocab), (rows, vocab + 1)):
        with pytest.raises(binding.ScoutError) as e:
            binding.scout_loss_workspace(dtype, more[0], 64, more[1])
        assert e.value.code == binding.ERR_UNSUPPORTED
