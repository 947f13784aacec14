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
