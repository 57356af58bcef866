"""What follows when a wait of the replay kernels gives up: the block ends, nothing is made again from what was not computed, and the
count says so."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stuck", [0, 0x01, 0x80, 0x10, 0x55, 0xFF])
def test_warps_that_gave_up_and_warps_that_did_not_leave_together(stuck):
    """Every warp leaves whoever gave up; rows are made again only if nobody did, each warp's own of both warpgroups."""
    from paper_2608_11034_b200 import binding
    assert binding.scout_replay_error() == 0
    out = torch.full((8, 2), 99, dtype=torch.int32, device="cuda")
    binding.scout_selftest_give_up(stuck, out.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    if stuck:
        assert out.tolist() == [[0, 0]] * 8
    else:
        assert out.tolist() == [[(1 << (w & 3)) | (1 << (4 + (w & 3))), 3] for w in range(8)]
    assert (binding.scout_replay_error() > 0) == (stuck != 0) and binding.scout_replay_error() == 0


def test_a_wait_that_gave_up_is_seen_by_everybody_who_looks():
    """One reader does not take the count from another, and results of such a call are refused before anybody votes on them."""
    from paper_2608_11034_b200 import binding, layer_replay, replay
    layer = layer_replay.make_layer(130, 264, 2, 1, 64)
    before = binding.scout_replay_waits()
    layer_replay.replay_layer(layer, layer.codes, layer.exps)
    assert binding.scout_replay_waits() == before
    out = torch.empty(16, dtype=torch.int32, device="cuda")
    with pytest.raises(replay.WaitGaveUp):
        with replay.waits_checked(torch.device("cuda")):
            binding.scout_selftest_give_up(1, out.data_ptr(), torch.cuda.current_stream().cuda_stream)
            with replay.waits_checked(torch.device("cuda")):
                pass
    now = binding.scout_replay_waits()
    assert now > before and binding.scout_replay_error() == now - before
    assert binding.scout_replay_waits() == now and binding.scout_replay_error() == 0
    with replay.waits_checked(torch.device("cuda")):          # and the next call is judged by itself
        layer_replay.replay_layer(layer, layer.codes, layer.exps)


def test_a_captured_replay_is_checked_where_the_graph_runs():
    from paper_2608_11034_b200 import layer_replay, replay
    layer = layer_replay.make_layer(130, 264, 2, 1, 64)
    want = layer_replay.replay_layer(layer, layer.codes, layer.exps)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer_replay.replay_layer(layer, layer.codes, layer.exps)
    with replay.waits_checked(torch.device("cuda")):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_refusals_of_the_selftest():
    from paper_2608_11034_b200 import binding
    for stuck, out in ((256, 256), (0, 0)):
        with pytest.raises(binding.ScoutError) as e:
            binding.scout_selftest_give_up(stuck, out, 0)
        assert e.value.code == binding.ERR_INVALID
