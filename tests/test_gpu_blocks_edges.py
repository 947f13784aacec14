"""Calls around a block's linears at the edges of what they accept, on the GPU, against the float64 oracle.  Bounds as in
test_gpu_blocks.py: n roundings of float32 leave n 2^-24 of the magnitudes behind a value, an output in bf16 another 2^-8 of itself."""
import pytest
import torch

from oracle import block_ops as ref
from paper_2503_06564_amd import trdq

pytestmark = pytest.mark.gpu


def dev():
    return torch.device("cuda:0")


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("params", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [1, 771, 4608])
def test_no_rows_have_zero_gradients(c, params):
    """Every parameter's gradient of a call without rows is written, also where a captured graph replays it."""
    none = torch.empty(0, c, dtype=torch.bfloat16, device=dev())
    vec, mods = torch.full((c,), float("nan"), dtype=params, device=dev()), torch.ones(3, 3 * c, dtype=params, device=dev())
    off = torch.zeros(4, dtype=torch.int32, device=dev())
    grads = {k: torch.empty(c, device=dev()) for k in ("dpre_weight", "dpre_bias", "dpost_weight", "dpost_bias")}
    grads.update({k: torch.empty(3, c, device=dev()) for k in ("dscale", "dshift", "dgate")})

    def call():
        trdq.block_norm_bwd(none, none, none, none, Y=none, pre_weight=vec, pre_bias=vec, post="layer", post_weight=vec, post_bias=vec,
                            shift=mods[:, :c], scale=mods[:, c:2 * c], gate=mods[:, 2 * c:], seg_off=off, **grads)

    def check():
        torch.cuda.synchronize()
        for k, g in grads.items():
            assert bool((g == 0).all()), k
            g.fill_(9.0)

    for g in grads.values():
        g.fill_(9.0)
    call()
    check()
    dgate = torch.full((c,), 9.0, device=dev())
    trdq.block_norm_bwd(none, none, none, none, Y=none, gate=vec, dgate=dgate, seg_len=7)
    torch.cuda.synchronize()
    assert bool((dgate == 0).all())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        graph.replay()
        check()


@pytest.mark.parametrize("off", [[0, 0, 9, 9, 20, 20], [0, 20, 20], [0, 0, 20]])
@pytest.mark.parametrize("c,post", [(96, None), (771, "layer"), (2304, "rms")])
def test_parameters_of_empty_segments_reach_nothing(off, c, post):
    """NaN and Inf in the scale, shift and gate of a segment without rows: the same outputs and gradients as with zeros there, zeros as
    its own gradients, also where a weight is not finite."""
    rows, segs = off[-1], len(off) - 1
    empty = torch.tensor([off[i] == off[i + 1] for i in range(segs)])
    seg_off = torch.tensor(off, dtype=torch.int32, device=dev())
    x, y, dxo, dh = ((rand(i, rows, c)).to(dev()).to(torch.bfloat16) for i in range(4))
    vec = {"pre_weight": rand(5, c), "pre_bias": rand(6, c)}
    if post:
        vec.update(post_weight=rand(7, c), post_bias=rand(8, c))
    vec["pre_weight"][3] = float("inf")
    vec = {k: v.to(dev()) for k, v in vec.items()}

    def run(mods):
        p = dict(vec, shift=mods[:, :c], scale=mods[:, c:2 * c], gate=mods[:, 2 * c:])
        xo, h, dx, dy = (torch.empty_like(x) for _ in range(4))
        grads = {"d" + k: torch.full(v.shape, 9.0, device=dev()) for k, v in p.items()}
        kw = dict(post=post, seg_off=seg_off, **p)
        trdq.block_norm(x, xo, h, Y=y, **kw)
        ws = torch.empty(trdq.block_norm_bwd_ws_nbytes(rows, c, segs), dtype=torch.uint8, device=dev())
        trdq.block_norm_bwd(dx, dy, xo, dh, Y=y, dXout=dxo, ws=ws, **grads, **kw)
        torch.cuda.synchronize()
        return dict(grads, xo=xo, h=h, dx=dx, dy=dy)

    mods = rand(9, segs, 3 * c) * 0.3
    mods[empty] = 0.0
    clean = run(mods.to(dev()))
    for bad in (float("nan"), float("inf")):
        mods[empty] = bad
        got = run(mods.to(dev()))
        for k in clean:
            assert torch.equal(got[k].nan_to_num(), clean[k].nan_to_num()) and torch.equal(got[k].isnan(), clean[k].isnan()), k
        for k in ("dscale", "dshift", "dgate"):
            assert bool((got[k].cpu()[empty] == 0).all()), k
        assert bool(got["dpre_bias"].isfinite().all())
