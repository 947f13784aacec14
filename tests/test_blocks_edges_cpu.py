"""Calls around a block's linears at the edges of what they accept, without a GPU: what is refused, and sizes that the library computes on
the host.  (Without a device a call whose arguments are right ends in ERR_HIP: nothing can be launched.)"""
import ctypes as C

import pytest
import torch

from paper_2503_06564_amd import trdq

X = torch.zeros(6, 40, dtype=torch.bfloat16)
WS = torch.zeros(1 << 20, dtype=torch.uint8)


def status(f, *args, **kw):
    """The status of a call whose tensors lie on the host; never run where a device could be handed their addresses."""
    with pytest.raises(trdq.TrdqError) as e:
        f(*args, stream=0, **kw)
    return e.value.status


def accepted():
    """What a call with right arguments answers here: host tensors are refused where there is a device."""
    return trdq.ERR_MISMATCH if torch.cuda.is_available() else trdq.ERR_HIP


def test_gate_of_one_row_has_no_gradient_per_segment():
    """An expanded vector reads as a gate, but [segments, c] cannot be its gradient: the library takes a gate without a row stride for
    one vector."""
    gate, kw = torch.ones(40).expand(3, 40), dict(Y=X, seg_len=2, ws=WS)
    for d in (torch.zeros(3, 40), torch.zeros(40)):
        assert status(trdq.block_norm_bwd, X, X, X, X, gate=gate, dgate=d, **kw) == trdq.ERR_SHAPE
    off = torch.tensor([0, 1, 4, 6], dtype=torch.int32)
    assert status(trdq.block_norm_bwd, X, X, X, X, gate=gate, dgate=torch.zeros(3, 40), Y=X, seg_off=off, ws=WS) == trdq.ERR_SHAPE
    # the gate itself, its gradient not asked for, a vector's and a matrix' own gradients: as before
    assert status(trdq.block_norm, X, X, X, Y=X, gate=gate, seg_len=2) == accepted()
    assert status(trdq.block_norm_bwd, X, X, X, X, gate=gate, **kw) == accepted()
    assert status(trdq.block_norm_bwd, X, X, X, X, gate=gate[0], dgate=torch.zeros(40), **kw) == accepted()
    assert status(trdq.block_norm_bwd, X, X, X, X, gate=gate.contiguous(), dgate=torch.zeros(3, 40), **kw) == accepted()
    assert status(trdq.block_norm_bwd, X, X, X, X, gate=gate[:1], dgate=torch.zeros(1, 40), Y=X, ws=WS) == accepted()


def test_no_rows_still_write_gradients():
    """A sum over no rows is zero, and is written: only a call that has no gradient to write returns without a launch."""
    none = X[:0]
    vec, grad = torch.ones(40), torch.full((40,), 9.0)
    trdq.block_norm_bwd(none, None, none, none, stream=0)
    trdq.block_norm_bwd(none, None, none, none, pre_weight=vec, scale=torch.ones(1, 40), stream=0)
    if torch.cuda.is_available():
        return                                              # (tests/test_gpu_blocks_edges.py holds the values)
    mods = torch.ones(3, 40)
    off = torch.zeros(4, dtype=torch.int32)
    assert status(trdq.block_norm_bwd, none, None, none, none, pre_weight=vec, dpre_weight=grad) == trdq.ERR_HIP
    assert status(trdq.block_norm_bwd, none, none, none, none, Y=none, post="rms", post_weight=vec, dpost_weight=grad) == trdq.ERR_HIP
    assert status(trdq.block_norm_bwd, none, none, none, none, Y=none, gate=vec, dgate=grad, seg_len=5) == trdq.ERR_HIP
    for name in ("scale", "shift", "gate"):
        kw = {name: mods, "d" + name: torch.full((3, 40), 9.0), "seg_off": off}
        assert status(trdq.block_norm_bwd, none, none, none, none, Y=none, **kw) == trdq.ERR_HIP
        trdq.block_norm_bwd(none, none, none, none, Y=none, seg_len=5, stream=0, **{name: mods[:0], "d" + name: mods[:0]})     # no segment either
        assert status(trdq.block_norm_bwd, none, None, none, none, **{"d" + name: grad[None] if name != "gate" else grad}) == trdq.ERR_NULL


def test_workspaces_own_what_they_count():
    """An expanded or strided workspace owns fewer bytes than it has elements, or not those that lie behind its address."""
    vec = dict(pre_weight=torch.ones(40), dpre_weight=torch.zeros(40))
    a, b = (torch.zeros(n, 4608, dtype=torch.uint8).view(torch.float8_e4m3fn) for n in (300, 1152))
    sa, sb, y = torch.ones(36, 300), torch.ones(36, 1152), torch.zeros(300, 1152)
    need = trdq.fp8_gemm_ws_nbytes(300, 1152, 4608)
    assert need > 0
    for n, f, args, kw in ((trdq.block_norm_bwd_ws_nbytes(6, 40, 1), trdq.block_norm_bwd, (X, None, X, X), vec),
                           (need, trdq.fp8_gemm, (a, sa, b, sb, y), {})):
        whole = torch.zeros(2 * n, dtype=torch.uint8)
        for ws in (whole[:1].expand(n), whole[::2], whole[:n].view(2, n // 2).t()):
            assert ws.numel() >= n and status(f, *args, ws=ws, **kw) == trdq.ERR_SHAPE
        assert status(f, *args, ws=whole[:n - 1], **kw) == trdq.ERR_SHAPE
        assert status(f, *args, ws=whole[:n], **kw) == accepted()
        assert status(f, *args, ws=whole[:n].view(torch.float32)[None], **kw) == accepted()


@pytest.mark.parametrize("seg_len", [6, 7, 2 ** 31, 2 ** 62, 2 ** 63 - 6, 2 ** 63 - 2, 2 ** 63 - 1])
def test_segments_longer_than_the_rows(seg_len):
    """One segment, however long it could be; its workspace is that of one segment."""
    mods, grad = torch.ones(1, 40), torch.zeros(1, 40)
    need = trdq.block_norm_bwd_ws_nbytes(6, 40, 1)
    assert status(trdq.block_norm, X, None, X, scale=mods, seg_len=seg_len) == accepted()
    args = (X, None, X, X)
    assert status(trdq.block_norm_bwd, *args, scale=mods, dscale=grad, seg_len=seg_len, ws=WS[:need]) == accepted()
    assert status(trdq.block_norm_bwd, *args, scale=mods, dscale=grad, seg_len=seg_len, ws=WS[:need - 4]) == trdq.ERR_SHAPE
    assert status(trdq.block_norm_bwd, *args, pre_weight=mods[0], dpre_weight=grad[0], seg_len=seg_len, ws=WS[:need - 4]) == trdq.ERR_SHAPE


@pytest.mark.parametrize("borders", [0, 1])
def test_borders_of_no_segment_are_refused(borders):
    off = torch.zeros(borders, dtype=torch.int32)
    for x in (X, X[:0]):
        assert status(trdq.block_norm, x, None, x, seg_off=off) == trdq.ERR_RANGE
        assert status(trdq.block_norm, x, None, x, scale=torch.ones(1, 40), seg_off=off) == trdq.ERR_RANGE
        assert status(trdq.block_norm_bwd, x, None, x, x, seg_off=off) == trdq.ERR_RANGE


@pytest.mark.parametrize("c", [1, 600, 1152, 4608, 16384])
def test_workspace_of_norm_gradients_is_bounded(c):
    """At most 512 runs (and as many as rows) beside the segments, four float32 sums each, up to the last row count that is accepted."""
    for rows in (1, 7, 8, 9, 511, 512, 513, 4095, 4097, 2 ** 20 + 1, 2 ** 30 + 3, 2 ** 31 - 4096, 2 ** 31 - 1000, 2 ** 31 - 300, 2 ** 31 - 258):
        for segments in (1, 2, 64, 4096, 2 ** 31 - 1):
            need = trdq.block_norm_bwd_ws_nbytes(rows, c, segments)
            assert (1 + segments) * 16 * c <= need <= (min(rows, 512) + segments) * 16 * c, (rows, segments)
    # sizes that no call takes
    for rows, width, segments in ((2 ** 31 - 256, c, 1), (0, c, 1), (5, 16385, 1), (5, c, 0), (5, c, 2 ** 31), (5, c, 2 ** 63 - 1)):
        assert trdq.block_norm_bwd_ws_nbytes(rows, width, segments) == 0


def test_most_rows():
    """Fewer than 2^31 - 256 rows are taken (a call without addresses gets as far as ERR_NULL), that many are not."""
    L, norm = trdq.lib(), trdq._Norm(c=40, x_dtype=trdq.BF16, param_dtype=trdq.F32, pre=1, post=0, eps=1e-6)
    calls = {
        "fp8_quant": lambda rows: L.trdq_fp8_quant(None, trdq.BF16, rows, 40, 40, 0, trdq.E4M3, None, 128, trdq.F32, None, rows, None),
        "fp8_gemm": lambda rows: L.trdq_fp8_gemm(rows, 40, 128, None, trdq.E4M3, 128, None, rows, None, trdq.E4M3, 128, None, 40, 0, trdq.F32, None, None,
                                                 trdq.BF16, 40, None, 0, None),
        "block_norm": lambda rows: L.trdq_block_norm(C.byref(norm), None, 40, None, 0, None, 0, trdq.BF16, None, 40, 0, None, 0, None),
        "block_norm_bwd": lambda rows: L.trdq_block_norm_bwd(C.byref(norm), C.byref(trdq._NormGrads()), None, 0, None)}
    for name, call in calls.items():
        for rows, want in ((2 ** 31 - 257, trdq.ERR_NULL), (2 ** 31 - 256, trdq.ERR_UNSUPPORTED)):
            norm.rows = rows
            assert call(rows) == want, (name, rows)
    assert trdq.block_norm_bwd_ws_nbytes(2 ** 31 - 257, 40, 1) > 0


def test_one_workspace_for_smaller_products():
    """Fewer rows may need a larger workspace (K is split further): one that is made for the largest sizes has a query of its own."""
    own, upto = trdq.fp8_gemm_ws_nbytes, trdq.fp8_gemm_ws_nbytes_upto
    assert any(own(m, 1152, 4608) > own(4096, 1152, 4608) for m in range(1, 4096))
    g = torch.Generator().manual_seed(1)
    draw = lambda n: int(torch.exp(torch.rand((), generator=g) * torch.log(torch.tensor(float(n)))))  # noqa: E731
    for M, N, K in ((4096, 1152, 4608), (8192, 4608, 1152), (4608, 1152, 8192), (300, 500, 640), (17, 64, 16384), (2100, 2200, 4224), (32768, 8192, 8192),
                    (2 ** 31 - 257, 128, 128)):
        most = upto(M, N, K)
        assert own(M, N, K) <= most <= 64 << 20
        for _ in range(400):
            m, n, k = draw(M), draw(N), -(-draw(K) // 128) * 128
            assert own(m, n, k) <= most and own(m, N, K) <= most and upto(m, n, k) <= most, (m, n, k)
        for m in range(1, min(M, 3000), 7):
            assert own(m, N, K) <= most, m
    assert upto(0, 128, 1024) == 0 and upto(128, 0, 1024) == 0 and upto(128, 128, 0) == 0 and upto(128, 128, 896) == 0
    for bad in ((2 ** 31, 128, 1024), (-1, 128, 1024)):
        assert upto(*bad) == 0


def test_training_takes_a_step_at_least():
    from paper_2503_06564_amd import fp8_block
    for steps in (0, -1):
        with pytest.raises(ValueError, match="steps"):
            fp8_block.train(128, 128, 1, steps)
