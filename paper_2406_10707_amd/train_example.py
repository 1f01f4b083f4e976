"""A small training run with the optimizer and the 4-bit operators of include/ckpt_train.h, next to what the library is for: two linear layers trained on a fixed linear target in 4-bit products with 8-bit moments,
snapshots while it goes on, and a restart from the first of them that ends in the same bits.

    python -m paper_2406_10707_amd.train_example [--steps 60] [--every 20] [--dir /dev/shm/...]

A step: master weights -> 4-bit copies by rows and by columns (never stored: the snapshot holds 6.06 bytes a parameter, master weights and 8-bit moments); forward h = x W1^T,
y - t = h W2^T - t (the product is added to -t); backward dW2 = (y - t)^T h, dh = (y - t) W2, dW1 = dh^T x, with the gradients of activations rounded stochastically; norm of both weight
gradients; wait for the end of the pending snapshot's window; clipped AdamW step; snapshot."""
import argparse
import tempfile

import numpy as np

from . import binding as B
from . import harness

TOKENS, INPUT, HIDDEN, OUTPUT = 1000, 320, 200, 96       # odd on purpose: no size has to be a multiple of anything


class Matrix4:
    """A 4-bit matrix with memory of its own."""

    def __init__(self, rows, cols):
        code_pitch, scale_pitch = B.mx_layout(B.CKPT_MXFP4, rows, cols)
        self.codes, self.scales = harness.DevBuf(rows * code_pitch), harness.DevBuf(rows * scale_pitch)
        self.mx = B.mx_matrix(B.CKPT_MXFP4, rows, cols, self.codes.ptr, code_pitch, self.scales.ptr, scale_pitch)


class Both:
    """A rows x cols f32 matrix in the two forms that products contract over."""

    def __init__(self, rows, cols):
        self.by_row, self.by_col = Matrix4(rows, cols), Matrix4(cols, rows)
        self.cols = cols

    def take(self, src, stream, stochastic=False, seed=0):
        B.mx_quantize(src.ptr, B.CKPT_F32, self.cols, self.by_row.mx, self.by_col.mx, stream, seed=seed,
                      rounding=B.CKPT_ROUND_STOCHASTIC if stochastic else B.CKPT_ROUND_NEAREST)


class Run:
    def __init__(self, directory, seed=1):
        rng = np.random.default_rng(seed)
        self.stream = harness.make_compute_stream()
        self.layers = [(HIDDEN, INPUT), (OUTPUT, HIDDEN)]
        self.weights = [self._upload((rng.standard_normal(s) / s[1] ** 0.5).astype(np.float32)) for s in self.layers]
        self.grads = [harness.DevBuf(4 * r * c) for r, c in self.layers]
        self.moments = [[self._upload(np.zeros(n, np.uint8)) for n in (r * c, r * c, -(-r * c // 32), -(-r * c // 32))] for r, c in self.layers]
        x = rng.standard_normal((TOKENS, INPUT)).astype(np.float32)
        target = x @ (rng.standard_normal((INPUT, OUTPUT)) / INPUT ** 0.5).astype(np.float32)
        self.x, self.minus_t = self._upload(x), self._upload(-target)
        self.h, self.dy, self.dh = (harness.DevBuf(4 * TOKENS * n) for n in (HIDDEN, OUTPUT, HIDDEN))
        self.x4, self.h4, self.dy4, self.dh4 = Both(TOKENS, INPUT), Both(TOKENS, HIDDEN), Both(TOKENS, OUTPUT), Both(TOKENS, HIDDEN)
        self.w4 = [Both(r, c) for r, c in self.layers]
        self.norm = harness.DevBuf(24)
        shapes = [(TOKENS, HIDDEN, INPUT), (TOKENS, OUTPUT, HIDDEN), (OUTPUT, HIDDEN, TOKENS), (TOKENS, HIDDEN, OUTPUT), (HIDDEN, INPUT, TOKENS)]
        self.workspace = harness.DevBuf(max(16, *(B.mx_gemm_workspace(*s) for s in shapes)))
        self.optimizer = B.Optimizer(
            [dict(numel=r * c, grad=g.ptr, master=w.ptr, m=s[0].ptr, v=s[1].ptr, m_scale=s[2].ptr, v_scale=s[3].ptr, weight_decay=0.01)
             for (r, c), w, g, s in zip(self.layers, self.weights, self.grads, self.moments)], grad_dtype=B.CKPT_F32, param_dtype=0, state_bits=8)
        self.x4.take(self.x, self.stream.cuda_stream)
        self.snapshots = B.Checkpointer(B.make_config(out_dir=directory, dma_chunk_bytes=256 << 10, pack_superchunk_bytes=1 << 20, host_ring_bytes=2 << 20))
        descs = []
        for k, ((r, c), w, s) in enumerate(zip(self.layers, self.weights, self.moments)):
            descs.append((f"layer{k}.master", B.CKPT_F32, (r, c), w.ptr, 4 * r * c))
            descs += [(f"layer{k}.{name}", B.CKPT_U8, (b.nbytes,), b.ptr, b.nbytes) for name, b in zip(("m", "v", "m_scale", "v_scale"), s)]
        self.snapshots.register_tensors(descs)
        self.state = [b for w, s in zip(self.weights, self.moments) for b in (w, *s)]

    @staticmethod
    def _upload(a):
        buf = harness.DevBuf(a.nbytes)
        buf.upload(a)
        return buf

    def _product(self, a, b, c, columns, accumulate=False):
        B.mx_gemm(a.mx, b.mx, c.ptr, B.CKPT_F32, columns, self.stream.cuda_stream, accumulate=accumulate, workspace=self.workspace.ptr, workspace_bytes=self.workspace.nbytes)

    def step(self, n):
        st = self.stream.cuda_stream
        for w4, w in zip(self.w4, self.weights):
            w4.take(w, st)
        (w1, w2), (g1, g2) = self.w4, self.grads
        self._product(self.x4.by_row, w1.by_row, self.h, HIDDEN)
        self.h4.take(self.h, st)
        B.proxy_copy_d2d_async(self.dy.ptr, self.minus_t.ptr, self.dy.nbytes, st)
        self._product(self.h4.by_row, w2.by_row, self.dy, OUTPUT, accumulate=True)
        self.dy4.take(self.dy, st, stochastic=True, seed=2 * n)
        self._product(self.dy4.by_col, self.h4.by_col, g2, HIDDEN)
        self._product(self.dy4.by_row, w2.by_col, self.dh, HIDDEN)
        self.dh4.take(self.dh, st, stochastic=True, seed=2 * n + 1)
        self._product(self.dh4.by_col, self.x4.by_col, g1, INPUT)
        self.optimizer.grad_norm(self.norm.ptr, st, max_norm=1.0, grad_scale=1.0 / TOKENS)
        self.snapshots.wait_immutable_window_end(st)      # before anything mutates the state
        self.optimizer.step(st, step=n, lr=3e-3, beta1=0.9, beta2=0.95, seed=7, stochastic=True, norm=self.norm.ptr)

    def loss(self):
        self.stream.synchronize()
        return float(np.mean(self.dy.download().view(np.float32).astype(np.float64) ** 2))

    def bits(self):
        self.stream.synchronize()
        return [b.download() for b in self.state]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--every", type=int, default=20)
    ap.add_argument("--dir", default=None, help="directory of the snapshots (default: a temporary one)")
    args = ap.parse_args(argv)
    with tempfile.TemporaryDirectory() as temporary:
        run = Run(args.dir or temporary)
        losses = []
        for n in range(1, args.steps + 1):
            run.step(n)
            if n % args.every == 0:
                run.snapshots.snapshot_async(n, run.stream.cuda_stream)
            if n == 1 or n % args.every == 0:
                losses.append(run.loss())
                print(f"step {n}: loss {losses[-1]:.5f}", flush=True)
        run.snapshots.flush()
        layout, last = run.snapshots.layout(), run.bits()
        parameters = sum(r * c for r, c in run.layers)
        print(f"snapshot: {layout['payload_bytes'] / parameters:.2f} bytes a parameter")
        if args.steps > args.every:
            for b in run.state:
                B.proxy_device_fill_async(b.ptr, 0xEE, b.nbytes, run.stream.cuda_stream)
            first = run.snapshots.restore(run.snapshots.file_name(args.every), run.stream.cuda_stream)
            for n in range(first + 1, args.steps + 1):
                run.step(n)
            same = all(np.array_equal(a, b) for a, b in zip(last, run.bits()))
            print(f"restarted from step {first}: the state after step {args.steps} is {'the same, bit for bit' if same else 'DIFFERENT'}")
            if not same:
                return 1
        run.snapshots.destroy()
        return 0 if losses[-1] < losses[0] else 1


if __name__ == "__main__":
    raise SystemExit(main())
