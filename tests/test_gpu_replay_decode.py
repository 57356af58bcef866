"""Attention of one or a few new tokens over long caches, as serving and the replay of a decoded step use it: sequences of every
length in one padded batch, padding that holds anything, keys in a few parts (one cluster) or in many (joined in a second launch),
many sequences, and caches whose offsets pass 32 bits."""
import math

import pytest
import torch

import replay_defn as defn

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def no_wait_gives_up():
    yield
    from paper_2608_11034_b200 import binding
    assert binding.scout_replay_error() == 0


def make(seed, dtype, B, Tq, Tk, Hq, Hk, D):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)          # noqa: E731
    return n(B, Tq, Hq, D), n(B, Tk, Hk, D), n(B, Tk, Hk, D)


def check(q, k, v, **kw):
    from paper_2608_11034_b200 import replay
    o, lse = replay.attention_forward(q, k, v, **kw)
    want = defn.attention(q, k, v, **kw)
    assert torch.isfinite(o).all() and ((o.double() - want["o"]).abs() <= want["b_o"]).all()
    empty = torch.isinf(want["lse"])
    assert torch.equal(empty, lse == -math.inf)
    assert ((lse.double() - want["lse"])[~empty].abs() <= 1e-5 * (1 + want["lse"][~empty].abs())).all()
    again = replay.attention_forward(q, k, v, **kw)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


SIZES = [  # B, Tq, Tk, Hq, Hk, D, causal, window
    (8, 1, 777, 32, 8, 128, True, 0),        # parts of a cluster
    (6, 2, 513, 8, 1, 64, True, 0),
    (5, 4, 300, 4, 1, 80, True, 70),
    (7, 1, 200, 16, 1, 8, False, 0),
    (5, 3, 1030, 15, 3, 120, True, 1),
    (1, 1, 8192, 32, 8, 128, True, 0),       # 55 parts, joined
    (2, 4, 4001, 4, 1, 64, True, 0),         # 31
    (1, 2, 5000, 2, 1, 96, False, 0),
    (3, 1, 3000, 2, 2, 128, True, 900),
    (40, 1, 150, 8, 8, 64, True, 0),         # one part
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_padded_caches(size, dtype):
    B, Tq, Tk, Hq, Hk, D, causal, window = size
    q, k, v = make(51, dtype, B, Tq, Tk, Hq, Hk, D)
    check(q, k, v, causal=causal, window=window)
    some = [Tk, 1, 0, Tq, 64, 65, Tk - 1, Tk // 2 + 3]
    for turn in range(min(B, 2) if B < 4 else 1):
        n = [min(Tk, some[(b + turn * B) % len(some)]) for b in range(B)]
        kb, vb = k.clone(), v.clone()
        for b in range(B):
            kb[b, n[b]:], vb[b, n[b]:] = math.nan, (math.inf if b % 2 else math.nan)
        lens = torch.tensor(n, dtype=torch.int32, device="cuda")
        check(q, kb, vb, causal=causal, window=window, kv_lens=lens)
        if Tq > 1:
            m = torch.tensor([(Tq - b) % (Tq + 1) for b in range(B)], dtype=torch.int32, device="cuda")
            qb = q.clone()
            for b in range(B):
                qb[b, int(m[b]):] = math.nan
            check(qb, kb, vb, causal=causal, window=window, q_lens=m, kv_lens=lens)


@pytest.mark.parametrize("Tq,Hq", [(1, 4), (1, 1), (33, 2), (128, 2)])
def test_offsets_beyond_32_bits(Tq, Hq):
    """A cache whose last tokens lie beyond 2^32 elements from its start, for keys and values, in every kernel."""
    from paper_2608_11034_b200 import replay
    T, D = 300, 64
    stride = (1 << 32) // (T - 100) // 8 * 8
    room = torch.empty((T - 1) * stride + 2 * D, dtype=BF, device="cuda")
    k, v = (room.as_strided((1, T, 1, D), (room.numel() // 8 * 8, stride, D, 1), at) for at in (0, D))
    q, ks, vs = make(52, BF, 1, Tq, T, Hq, 1, D)
    k.copy_(ks), v.copy_(vs)
    got, want = replay.attention_forward(q, k, v, causal=True), replay.attention_forward(q, ks, vs, causal=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check(q, ks, vs, causal=True)


@pytest.mark.parametrize("T", [1, 3, 20, 100])
def test_more_sequences_than_a_grid_axis_holds(T):
    """70000 sequences: looked at singly here and there, the results are those of the definition; forward and backward."""
    from paper_2608_11034_b200 import replay
    B, H, D = 70000, 1, 8
    q, k, v = make(53, BF, B, T, T, H, H, D)
    do = make(54, BF, B, T, T, H, H, D)[0]
    o, lse = replay.attention_forward(q, k, v, causal=True)
    dq, dk, dv = replay.attention_backward(q, k, v, o, lse, do, causal=True)
    some = [0, 1, 32767, 32768, 65535, 65536, 69999]
    want = defn.attention(q[some], k[some], v[some], do[some], causal=True)
    for name, got in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert torch.isfinite(got).all() and ((got[some].double() - want[name]).abs() <= want["b_" + name]).all(), name
    assert ((lse[some].double() - want["lse"]).abs() <= 1e-5 * (1 + want["lse"].abs())).all()
