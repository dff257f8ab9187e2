"""GPU tests of the products over row groups at sizes that take few-row, 128 and 256 wide tiles, whole and with split
depths, against the 64-bit oracle (every kind of tile in every product, by exact sums: test_gpu_block_sums.py); and of
calls that run at the same time."""
import numpy as np
import pytest
import torch

from tests import blocks as K
from tests.test_gpu_ffn import B, Block, verify  # noqa: F401  (B is the fixture)
from tests.test_gpu_int8 import Gemm, rows_bf16

pytestmark = pytest.mark.gpu


def sums(B, b, backward):
    """Bytes of partial sums in a block's workspace: none where no product is split."""
    planes = (3 if backward else 1) * ((b.T * b.F * 2 + 255) // 256 * 256)
    return B.moe_ffn_workspace_size(b.cfg, backward) - planes - 256


# whole 256-row tiles fill the chip: one and more stages, both widths, rows that end inside a tile
@pytest.mark.parametrize("T,H,F,G,off", [(8192, 64, 1024, 1, None), (8192, 1024, 64, 1, None), (8190, 192, 1024, 1, None),
                                         (8190, 1024, 320, 1, None), (9000, 256, 960, 3, [5, 4100, 4101, 8999])])
def test_large_tiles(B, T, H, F, G, off):
    verify(Block(T, H, F, G, off, "silu", seed=21).cuda(B))


# 128-row tiles, the depth of each product in several parts
@pytest.mark.parametrize("T,H,F", [(300, 2048, 4096), (290, 4096, 2112)])
def test_small_tiles_in_parts(B, T, H, F):
    b = Block(T, H, F, 1, None, "gelu", seed=22).cuda(B)
    assert sums(B, b, False) > 0 and sums(B, b, True) > 0
    verify(b)


# few rows, the depth of the second or of the first product in several parts
@pytest.mark.parametrize("T,H,F,G,off", [(5, 64, 8192, 1, None), (5, 8256, 64, 1, None), (33, 128, 7168, 2, [0, 1, 32])])
def test_few_rows_in_parts(B, T, H, F, G, off):
    b = Block(T, H, F, G, off, "silu", seed=23).cuda(B)
    assert sums(B, b, False) > 0
    verify(b)


# weights' gradients of few tiles over many rows: the rows in several parts, of groups that differ in depth
@pytest.mark.parametrize("T,off", [(3000, [0, 3000]), (3001, [0, 1, 2987]), (2500, [0, 0, 2490, 2491])])
def test_weight_gradients_in_parts(B, T, off):
    b = Block(T, 64, 64, len(off) - 1, off, "silu", seed=24).cuda(B)
    assert sums(B, b, True) > 0
    verify(b)


@pytest.mark.parametrize("T,D,N,G,off,act", [(8192, 128, 2048, 1, None, "silu"), (8190, 192, 1032, 1, None, "none"),
                                             (9000, 448, 1920, 3, [5, 4100, 4101, 8999], "gelu"),
                                             (300, 4160, 272, 1, None, "silu"), (5, 28736, 144, 1, None, "silu"),
                                             (40, 16384, 200, 2, [1, 3, 39], "none")])
def test_products_of_every_plan(B, T, D, N, G, off, act):
    Gemm(B, T, D, N, G, off, act, seed=25).verify()


def test_calls_at_the_same_time(B):
    """Blocks on four streams, each with its own workspace, against the same ones run alone."""
    shapes = [(700, 256, 320, 3, [0, 300, 301, 700]), (5, 64, 8192, 1, None), (2048, 128, 512, 2, [0, 2000, 2048]),
              (3000, 64, 64, 1, None)]
    blocks = [Block(*s, "silu", seed=26 + i).cuda(B) for i, s in enumerate(shapes)]
    alone = []
    for b in blocks:
        (y, gate, up), _ = b.forward()
        alone.append((y, gate, up, b.backward(gate, up)[0]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(3):
        runs = []
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                fwd, _ = b.forward(stream=s)
                runs.append((*fwd, b.backward(fwd[1], fwd[2], stream=s)[0]))
        torch.cuda.synchronize()
        for a, r in zip(alone, runs):
            for x, y in zip(a[:3], r[:3]):
                assert torch.equal(x.view(torch.int16), y.view(torch.int16))
            for n in a[3]:
                assert torch.equal(a[3][n].view(torch.int16), r[3][n].view(torch.int16)), n


def test_weight_quantiser_replays(B):
    G, D, N = 3, 320, 192
    w = torch.empty(G, D, N, dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty(G, N, D, dtype=torch.int8, device="cuda"), torch.empty(G, N, device="cuda")
    w.copy_(rows_bf16(G * D, N, 1).view(G, D, N))
    B.moe_quantize_weights_i8(G, D, N, N, 0, w, q, s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.moe_quantize_weights_i8(G, D, N, N, 0, w, q, s)
    for turn in range(4):
        x = rows_bf16(G * D, N, turn).view(G, D, N) * 2.0 ** -turn
        w.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        eq, es = K.quantize_rows(x.float().transpose(1, 2).numpy())
        assert np.array_equal(q.cpu().numpy(), eq) and np.array_equal(s.cpu().numpy(), es), turn


@pytest.mark.parametrize("T,off", [(32, None), (64, None), (128, None), (256, None), (512, None), (132, [0, 33, 66, 99, 132]),
                                   (516, [0, 129, 258, 387, 516]), (259, [0, 1, 258, 259]), (98, [0, 33, 33, 98]),
                                   (5, [0, 1, 2, 3, 4, 5, 5, 5])])
def test_the_most_row_tiles_there_can_be(B, T, off):
    """Groups of whole tiles, and of one row more than whole tiles: each launch has a workgroup for every tile."""
    verify(Block(T, 128, 192, len(off) - 1 if off else 1, off, "silu", seed=27).cuda(B))
    Gemm(B, T, 192, 144, len(off) - 1 if off else 1, off, "silu", seed=28).verify()


@pytest.mark.parametrize("T,H,F", [(8192, 64, 1024), (8193, 64, 1024)])
def test_the_most_wide_row_tiles_there_can_be(B, T, H, F):
    verify(Block(T, H, F, 1, None, "silu", seed=29).cuda(B))
    b = Block(T, H, F, 3, [0, 2561, 5378, T], "silu", seed=30).cuda(B)
    verify(b)


def test_8_bit_calls_at_the_same_time(B):
    """Quantisers and products on streams of their own, each behind its own inputs and sentinels, against the same
    ones run alone: by the stream given, and by the current one."""
    shapes = [(700, 448, 320, 3, [0, 300, 301, 700], "silu"), (5, 28736, 144, 1, None, "silu"),
              (8190, 448, 528, 1, None, "none"), (40, 16384, 200, 2, [1, 3, 39], "none")]
    gemms = [Gemm(B, *s, seed=40 + i) for i, s in enumerate(shapes)]
    xs = [rows_bf16(s[0], s[1], 44 + i).cuda() for i, s in enumerate(shapes)]
    w = [rows_bf16(192 * (i + 1), 128, 48 + i).view(i + 1, 192, 128).cuda() for i in range(4)]

    def run(g, x, w, stream):
        B.moe_quantize_rows_i8(*x.shape, x, g.d[0], g.d[1], stream)
        wq, ws = torch.full((len(w), 128, 192), 99, dtype=torch.int8, device="cuda"), torch.full((len(w), 128), 9.0, device="cuda")
        B.moe_quantize_weights_i8(len(w), 192, 128, 128, 0, w, wq, ws, stream)
        return g.run(stream)[0], g.d[0].clone(), g.d[1].clone(), wq, ws

    alone = [run(*a, None) for a in zip(gemms, xs, w)]
    streams = [torch.cuda.Stream() for _ in gemms]
    torch.cuda.synchronize()
    for turn in range(4):
        runs = []
        for a, s in zip(zip(gemms, xs, w), streams):
            # fills and launches on one stream, so in order
            with torch.cuda.stream(s):
                runs.append(run(*a, s if turn % 2 else None))
        torch.cuda.synchronize()
        for a, r in zip(alone, runs):
            for p, q in zip(a, r):
                assert torch.equal(p.contiguous().view(torch.int8), q.contiguous().view(torch.int8))


def test_a_stream_that_waits_for_another(B):
    """Inputs and sentinels of the current stream, the calls on a given one that waits for it, and back."""
    b = Block(700, 256, 320, 3, [0, 300, 301, 700], "silu", seed=52).cuda(B)
    g = Gemm(B, 333, 448, 320, 3, [0, 100, 101, 333], "silu", seed=53)
    (y, gate, up), _ = b.forward()
    r, _ = b.backward(gate, up)
    y8, _ = g.run()
    torch.cuda.synchronize()
    s, here = torch.cuda.Stream(), torch.cuda.current_stream()
    out = {n: torch.full_like(t, 3.0) for n, t in dict(y=y, gate=gate, up=up, y8=y8, **r).items()}
    s.wait_stream(here)
    d = b.d
    B.moe_ffn_forward(b.cfg, d["x"], d["off"], d["w1"], d["w3"], d["w2"], out["gate"], out["up"], out["y"], b.ws, s)
    B.moe_ffn_backward(b.cfg, d["dy"], d["x"], d["off"], d["w1"], d["w3"], d["w2"], out["gate"], out["up"], out["dx"],
                       out["dw1"], out["dw3"], out["dw2"], b.ws, s)
    B.moe_gemm_i8(g.cfg, g.d[0], g.d[1], g.doff, g.d[2], g.d[3], out["y8"], g.ws, s)
    here.wait_stream(s)
    for n, t in dict(y=y, gate=gate, up=up, y8=y8, **r).items():
        assert torch.equal(out[n].view(torch.int16), t.view(torch.int16)), n
