"""The calls around a block's linears put together: the MLP half of a DiT block in 8-bit floating point, forward and backward.

    python -m paper_2503_06564_amd.fp8_block [--tokens 4096] [--width 1152] [--batch 16] [--steps 20]

trains one such half block on synthetic data and prints the loss and the time of a step:

    x' = x + gate y,  h = norm(x') (1 + scale) + shift             trdq.block_norm, one pass
    a = h W1 + b1,  u = gelu(a),  z = u W2 + b2                    trdq.fp8_quant, trdq.fp8_gemm (h and u become e4m3 codes)
    x' + gate2 z                                                   is the next block's trdq.block_norm

and back: output gradients become e5m2 codes, by rows for the input gradient and by columns for the weight gradient (float32).
Everything between is explicit: no autograd, every buffer the caller's, so a step can be captured into a graph."""
import argparse
import time

from . import trdq


def _up(n):
    return (n + trdq.BLOCK - 1) // trdq.BLOCK * trdq.BLOCK


def _codes(rows, k, fmt, device, tiles=False):
    """Buffers for codes [rows, up(k)] and their scales."""
    import torch
    kind = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    n = (rows + trdq.BLOCK - 1) // trdq.BLOCK if tiles else rows
    return torch.empty(rows, _up(k), dtype=torch.uint8, device=device).view(kind), torch.empty(_up(k) // trdq.BLOCK, n, device=device)


class Fp8Linear:
    """y = x W^T + b with W [out, in] float32, products of codes.  `tokens` is the most rows of x (fewer, or none, use the front of the
    buffers, all of which are made here)."""

    def __init__(self, W, b, tokens):
        import torch
        self.W, self.b, self.tokens = W, b, tokens
        out, inn = W.shape
        dev = W.device
        self.w, self.wt = _codes(out, inn, "e4m3", dev, tiles=True), _codes(inn, out, "e4m3", dev, tiles=True)
        self.xt, self.dy, self.dyt = _codes(inn, tokens, "e4m3", dev), _codes(tokens, out, "e5m2", dev), _codes(out, tokens, "e5m2", dev)
        self.dW, self.db = torch.empty_like(W), torch.empty_like(b)
        need = max(trdq.fp8_gemm_ws_nbytes_upto(tokens, out, _up(inn)), trdq.fp8_gemm_ws_nbytes_upto(tokens, inn, _up(out)),
                   trdq.fp8_gemm_ws_nbytes_upto(out, inn, _up(tokens)))
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
        self.ones = torch.ones(1, tokens, device=dev)
        self.set_weights()

    def set_weights(self):
        """Codes of the weights as they are now: 128 x 128 tiles, as they lie and transposed."""
        trdq.fp8_quant(self.W, *self.w, blocks="tiles")
        trdq.fp8_quant(self.W, *self.wt, blocks="tiles_t")

    def forward(self, codes, scales, y):
        trdq.fp8_gemm(codes, scales, *self.w, y, bias=self.b, ws=self.ws)

    def backward(self, x, dy, dx):
        """dx (bf16), dW and db from dy (bf16) and the input x (bf16)."""
        import torch
        rows = x.shape[0]
        if rows == 0:                                               # (a product has a block of K at least)
            self.dW.zero_()
            self.db.zero_()
            return
        by_rows = lambda c: (c[0][:rows], c[1][:, :rows])  # noqa: E731
        by_cols = lambda c: (c[0][:, :_up(rows)], c[1][:_up(rows) // trdq.BLOCK])  # noqa: E731
        dyq, dyt, xt = by_rows(self.dy), by_cols(self.dyt), by_cols(self.xt)
        trdq.fp8_quant(dy, *dyq, blocks="rows")
        trdq.fp8_gemm(*dyq, *self.wt, dx, ws=self.ws)
        trdq.fp8_quant(dy, *dyt, blocks="cols")
        trdq.fp8_quant(x, *xt, blocks="cols")
        trdq.fp8_gemm(*dyt, *xt, self.dW, ws=self.ws)
        torch.matmul(self.ones[:, :rows], dy.float(), out=self.db[None])      # (a sum over rows would clear memory in a captured graph)


class MlpBlock:
    """norm -> linear -> gelu -> linear of `tokens` rows of `width` channels in `batch` samples, with modulation [batch, 3 width]
    (shift, scale, gate) and the gated residual of the branch before it."""

    def __init__(self, tokens, width, batch, device="cuda", hidden=None, seed=0):
        import torch
        g = torch.Generator().manual_seed(seed)
        hidden = hidden or 4 * width
        rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.tokens, self.width, self.batch, self.seg_len = tokens, width, batch, -(-tokens // batch)
        self.fc1 = Fp8Linear((rand(hidden, width) * width ** -0.5).to(device), torch.zeros(hidden, device=device), tokens)
        self.fc2 = Fp8Linear((rand(width, hidden) * hidden ** -0.5).to(device), torch.zeros(width, device=device), tokens)
        self.mods = (rand(-(-tokens // self.seg_len), 3 * width) * 0.2).to(device)
        e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device=device)  # noqa: E731
        self.x, self.a, self.u, self.z = e(tokens, width), e(tokens, hidden), e(tokens, hidden), e(tokens, width)
        self.h, self.hq, self.uq = e(tokens, width), _codes(tokens, width, "e4m3", device), _codes(tokens, hidden, "e4m3", device)
        self.du, self.dh, self.dx, self.dy = e(tokens, hidden), e(tokens, width), e(tokens, width), e(tokens, width)
        segs = self.mods.shape[0]
        self.dmods = [torch.empty(segs, width, device=device) for _ in range(3)]
        self.ws = e(trdq.block_norm_bwd_ws_nbytes(tokens, width, segs), dt=torch.uint8)

    def _norm(self):
        c = self.width
        return dict(pre="layer", shift=self.mods[:, :c], scale=self.mods[:, c:2 * c], gate=self.mods[:, 2 * c:], seg_len=self.seg_len)

    def forward(self, x, y):
        """z of the stream x and the branch y before this one; self.x is the stream with the branch."""
        import torch
        trdq.block_norm(x, self.x, self.h, Y=y, **self._norm())
        trdq.fp8_quant(self.h, *self.hq)
        self.fc1.forward(*self.hq, self.a)
        self.u.copy_(torch.nn.functional.gelu(self.a.float()))
        trdq.fp8_quant(self.u, *self.uq)
        self.fc2.forward(*self.uq, self.z)
        return self.z

    def backward(self, y, dx, dz):
        """From the gradients of self.x (what passes the block by) and of z: self.dx, self.dy, the weights' and the modulations'."""
        import torch
        self.fc2.backward(self.u, dz, self.du)
        a = self.a.float()
        cdf = 0.5 * (1.0 + torch.erf(a * 0.5 ** 0.5))
        self.du.copy_(self.du.float() * (cdf + a * torch.exp(-0.5 * a * a) * 0.3989422804014327))
        self.fc1.backward(self.h, self.du, self.dh)
        trdq.block_norm_bwd(self.dx, self.dy, self.x, self.dh, Y=y, dXout=dx, dshift=self.dmods[0], dscale=self.dmods[1], dgate=self.dmods[2],
                            ws=self.ws, **self._norm())

    def step(self, rate):
        """Plain gradient descent."""
        for lin in (self.fc1, self.fc2):
            lin.W.sub_(lin.dW, alpha=rate)
            lin.b.sub_(lin.db, alpha=rate)
            lin.set_weights()
        for i, d in enumerate(self.dmods):
            self.mods[:, i * self.width:(i + 1) * self.width].sub_(d, alpha=rate)


def train(tokens, width, batch, steps, rate=2.0, seed=0):
    """Losses of `steps` steps towards a fixed random target, and the seconds of one."""
    if steps < 1:
        raise ValueError("steps: one at least")
    import torch
    g = torch.Generator().manual_seed(seed + 1)
    x, y, target = ((torch.randn(tokens, width, generator=g)).to("cuda").to(torch.bfloat16) for _ in range(3))
    block = MlpBlock(tokens, width, batch, seed=seed)
    losses, began = [], 0.0
    for i in range(steps):
        if i == min(3, steps - 1):
            torch.cuda.synchronize()
            began, first = time.perf_counter(), i
        z = block.forward(x, y)
        d = block.x.float() + z.float() - target.float()
        losses.append((d * d).mean())
        dz = (d * (2.0 / d.numel() * tokens)).to(torch.bfloat16)
        block.backward(y, dz, dz)
        block.step(rate / tokens)
    torch.cuda.synchronize()
    return [float(v) for v in losses], (time.perf_counter() - began) / (steps - first)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1152)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    losses, seconds = train(a.tokens, a.width, a.batch, a.steps)
    print("loss " + " ".join(f"{v:.4f}" for v in losses))
    print(f"{seconds * 1e3:.3f} ms a step ({a.tokens} tokens, width {a.width}, {a.batch} samples)")


if __name__ == "__main__":
    main()
