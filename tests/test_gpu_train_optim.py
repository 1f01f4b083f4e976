"""The gradient norm and the AdamW step over tensor lists against the oracle: moments bit for bit (each operation of theirs is a rounding that
the definition names), master weights within the bound of the update's f32 operations, the working copy the rounding of the master weights the step
left. Sizes from zero and one element on, unaligned starts, guards around every part."""
import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu

GUARD = 64
DTYPES = {"f32": (B.CKPT_F32, 4), "bf16": (B.CKPT_BF16, 2), "f16": (B.CKPT_F16, 2), None: (0, 0)}
SIZES = [1, 2, 31, 32, 33, 0, 100, 255, 256, 257, 1000, 4095, 4096, 4097, 16384, 20001, 3, 65537, 0, 130]


class Arena:
    """Parts of tensors in one allocation, 0xEE between them."""

    def __init__(self, nbytes):
        self.buf, self.used = harness.DevBuf(nbytes), 0
        self.host = np.full(nbytes, 0xEE, np.uint8)
        self.parts = []

    def add(self, data, align, shift):
        raw = np.ascontiguousarray(data).view(np.uint8).reshape(-1)
        at = (self.used + GUARD + 63) // 64 * 64 + align * shift
        self.host[at:at + raw.size] = raw
        self.used = at + raw.size
        self.parts.append((at, raw.size))
        assert self.used + GUARD <= self.buf.nbytes
        return self.buf.ptr + at

    def upload(self):
        self.buf.upload(self.host)

    def read(self, k):
        at, n = self.parts[k]
        return self.now[at:at + n]

    def fetch(self):
        self.now = gu.download(self.buf)
        outside = np.ones(self.now.size, bool)
        for at, n in self.parts:
            outside[at:at + n] = False
        assert np.all(self.now[outside] == 0xEE), "written outside the tensors"


def as_grad(x, dtype):
    return x.astype(np.float32) if dtype == "f32" else to.half_bits(x.astype(np.float32), dtype)


def grad_values(stored, dtype):
    return stored if dtype == "f32" else to.half_values(stored, dtype).astype(np.float32)


class Setup:
    def __init__(self, sizes, grad, param, bits, seed, special=False):
        rng = np.random.default_rng(seed)
        self.sizes, self.grad, self.param, self.bits = sizes, grad, param, bits
        self.arena = Arena(sum(sizes) * 20 + len(sizes) * 9 * 256 + 4096)
        self.state, tensors = [], []
        for k, n in enumerate(sizes):
            g = rng.standard_normal(n) * 10.0 ** rng.integers(-5, -1)
            m, v = 0.1 * rng.standard_normal(n) * 1e-3, (rng.standard_normal(n) * 1e-3) ** 2
            if special:
                for b in range(0, n, 32):
                    u = rng.random()
                    if u < 0.15:
                        g[b:b + 32] = m[b:b + 32] = v[b:b + 32] = 0
                    elif u < 0.3:
                        g[b:b + 32] *= 10.0 ** rng.uniform(-9, 0, g[b:b + 32].size)
                        v[b:b + 32] *= 10.0 ** rng.uniform(-12, 0, v[b:b + 32].size)
                    elif u < 0.35:
                        v[b:b + 32] = m[b:b + 32] = 0
            w = (0.02 * rng.standard_normal(n)).astype(np.float32)
            m, v = m.astype(np.float32), v.astype(np.float32)
            decay = [0.0, 0.1, 0.01][k % 3]
            s = dict(g=as_grad(g, grad), w=w, decay=decay)
            t = dict(numel=n, weight_decay=decay)
            index = {}

            def place(name, data, align):
                index[name] = len(self.arena.parts)
                t[name] = self.arena.add(data, align, (k + len(index)) % 4) if n else None
                if not n:
                    self.arena.parts.append((0, 0))

            place("grad", s["g"], DTYPES[grad][1])
            place("master", w, 4)
            if param:
                place("param", np.zeros(n, np.uint16), 2)
            if bits == 32:
                s["m"], s["v"] = m, v
                place("m", m, 4)
                place("v", v, 4)
            else:
                for name, x in (("m", m), ("v", v)):
                    c, b = to.moment8(x, nonzero=name == "v")
                    s[name] = to.values(c.reshape(1, -1), b.reshape(1, -1), to.MXFP8).reshape(-1).astype(np.float32)
                    place(name, c, 1)
                    place(name + "_scale", b, 1)
            s["index"] = index
            self.state.append(s)
            tensors.append(t)
        self.arena.upload()
        self.tensors = tensors
        self.opt = B.Optimizer(tensors, grad_dtype=DTYPES[grad][0], param_dtype=DTYPES[param][0], state_bits=bits)

    def part(self, k, name):
        return self.arena.read(self.state[k]["index"][name])

    def check(self, hyper, scale, seed=None):
        """The device's state is one step behind `state`'s."""
        self.arena.fetch()
        blocks = 0
        for k, (n, s) in enumerate(zip(self.sizes, self.state)):
            if n == 0:
                continue
            m, v = to.moments(s["m"], s["v"], grad_values(s["g"], self.grad), scale, hyper["beta1"], hyper["beta2"])
            if self.bits == 32:
                assert np.array_equal(self.part(k, "m").view(np.float32), m) and np.array_equal(self.part(k, "v").view(np.float32), v)
                s["m"], s["v"] = m, v
            else:
                rm, rv = (None, None) if seed is None else to.step_bits16(seed, hyper["step"], blocks, n)
                for name, x, r in (("m", m, rm), ("v", v, rv)):
                    c, b = to.moment8(x, r, nonzero=name == "v")
                    assert np.array_equal(self.part(k, name + "_scale"), b), (k, name)
                    assert np.array_equal(self.part(k, name), c), (k, name)
                    s[name] = to.values(c.reshape(1, -1), b.reshape(1, -1), to.MXFP8).reshape(-1).astype(np.float32)
                assert np.all((s["v"] > 0) | (v == 0))
            want, update = to.adamw(s["w"], m, v, hyper["lr"], hyper["beta1"], hyper["beta2"], hyper["eps"], hyper["step"], s["decay"])
            got = self.part(k, "master").view(np.float32)
            # keep's rounding, its product and the difference: 3 x 2^-24 of the weight; the update: lr, two corrections, two products,
            # the root's argument, root and quotient to 1 ulp, the sum with eps: under 16 x 2^-23 of it
            assert np.all(np.abs(got - want) <= 2.0 ** -22 * np.abs(s["w"]) + 2.0 ** -19 * update + 1e-38)
            if self.param:
                assert np.array_equal(self.part(k, "param").view(np.uint16), to.half_bits(got, self.param))
            s["w"] = got.copy()
            blocks += -(-n // 32)


@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("param,bits,stochastic", [("bf16", 32, False), (None, 32, False), ("f16", 8, False), ("bf16", 8, True), (None, 8, True), ("bf16", 8, False)])
def test_three_steps(grad, param, bits, stochastic):
    print(f"adamw grad {grad} param {param} bits {bits} stochastic {stochastic}", flush=True)
    s = Setup(SIZES, grad, param, bits, seed=bits + len(grad), special=True)
    for step in (1, 2, 1000):
        hyper = dict(lr=3e-4, beta1=0.9, beta2=0.95 if step < 1000 else 0.999, eps=1e-8, step=step)
        s.opt.step(0, seed=77, stochastic=stochastic, **hyper)
        harness.synchronize()
        s.check(hyper, 1.0, 77 if stochastic else None)


@pytest.mark.parametrize("bits", [32, 8])
def test_scale_and_skip_come_from_the_norm(bits):
    print(f"norm, clipped step and skipped step, {bits} bits", flush=True)
    s = Setup(SIZES, "f32", "bf16", bits, seed=3)
    norm = harness.DevBuf(24)
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=5)
    s.opt.grad_norm(norm.ptr, 0, max_norm=0.25, grad_scale=0.5)
    s.opt.step(0, norm=norm.ptr, **hyper)
    harness.synchronize()
    r = B.ckpt_norm_result.from_buffer_copy(gu.download(norm).tobytes())
    total = sum(float(np.sum(x["g"].astype(np.float64) ** 2)) for x in s.state)
    assert abs(r.sum_squares - total) <= 1e-12 * total and r.nonfinite == 0
    assert abs(r.norm - 0.5 * total ** 0.5) <= 2.0 ** -23 * r.norm
    assert 0.25 / (0.5 * total ** 0.5) < 1 and abs(r.scale - 0.5 * 0.25 / (0.5 * total ** 0.5)) <= 2.0 ** -23 * r.scale
    s.check(hyper, r.scale)
    for bad in (np.inf, -np.inf, np.nan):
        before = gu.download(s.arena.buf)
        k = len(SIZES) - 1
        at, _ = s.arena.parts[s.state[k]["index"]["grad"]]
        good = before[at + 4 * 77:at + 4 * 78].copy()
        x = np.array([bad], np.float32)
        B.proxy_copy_h2d(s.arena.buf.ptr + at + 4 * 77, x.ctypes.data, 4)
        changed = gu.download(s.arena.buf)
        s.opt.grad_norm(norm.ptr, 0, max_norm=1.0)
        s.opt.step(0, norm=norm.ptr, **hyper)
        harness.synchronize()
        r = B.ckpt_norm_result.from_buffer_copy(gu.download(norm).tobytes())
        assert r.nonfinite == 1 and r.scale == 0 and np.array_equal(gu.download(s.arena.buf), changed)
        B.proxy_copy_h2d(s.arena.buf.ptr + at + 4 * 77, good.ctypes.data, 4)
        s.opt.grad_norm(norm.ptr, 0)
        harness.synchronize()
        r = B.ckpt_norm_result.from_buffer_copy(gu.download(norm).tobytes())
        assert r.nonfinite == 0 and r.scale == 1


@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", [[1], [0, 3], [4096], [70000], [5] * 3000, [300000, 1, 99999, 64, 4097], [0]])
def test_norm(grad, sizes):
    print(f"norm {grad} of {len(sizes)} tensors", flush=True)
    rng = np.random.default_rng(len(sizes))
    arena = Arena(sum(sizes) * 4 + len(sizes) * 256 + 4096)
    tensors, total = [], 0.0
    for k, n in enumerate(sizes):
        g = as_grad(rng.standard_normal(n) * 10.0 ** rng.integers(-6, 3 if grad != "f32" else 25), grad)
        total += float(np.sum(grad_values(g, grad).astype(np.float64) ** 2))
        tensors.append(dict(numel=n, grad=arena.add(g, DTYPES[grad][1], k % 5) if n else None))
    arena.upload()
    opt = B.Optimizer(tensors, grad_dtype=DTYPES[grad][0])
    out = harness.DevBuf(24)
    results = []
    for _ in range(3):
        opt.grad_norm(out.ptr, 0, max_norm=1e9)
        harness.synchronize()
        results.append(gu.download(out).tobytes())
    assert len(set(results)) == 1
    r = B.ckpt_norm_result.from_buffer_copy(results[0])
    assert abs(r.sum_squares - total) <= 1e-12 * total and abs(r.norm - total ** 0.5) <= 2.0 ** -23 * total ** 0.5 and r.nonfinite == 0
    if total:
        want = min(1.0, 1e9 / total ** 0.5)
        assert abs(r.scale - want) <= 2.0 ** -23 * want
    if sum(sizes):
        with pytest.raises(B.CkptError) as e:
            opt.step(0, step=1, lr=1e-3)
        assert e.value.code == B.CKPT_ESTATE


def test_new_gradients():
    print("set_grads", flush=True)
    sizes = [100 + k % 7 for k in range(1000)]
    arena = Arena(2 * (sum(sizes) * 4 + len(sizes) * 256) + 4096)
    lists = [[arena.add(np.full(n, c + 1, np.float32), 4, 0) for n in sizes] for c in range(2)]
    arena.upload()
    opt = B.Optimizer([dict(numel=n, grad=p) for n, p in zip(sizes, lists[0])], grad_dtype=B.CKPT_F32)
    out = harness.DevBuf(24)
    for c in (0, 1, 0):
        opt.set_grads(lists[c], 0)
        opt.grad_norm(out.ptr, 0)
        harness.synchronize()
        assert B.ckpt_norm_result.from_buffer_copy(gu.download(out).tobytes()).sum_squares == (c + 1) ** 2 * sum(sizes)
    for bad in (lists[0][:-1], lists[0][:-1] + [None], lists[0][:-1] + [lists[0][-1] + 2]):
        with pytest.raises(B.CkptError):
            opt.set_grads(bad, 0)


def test_two_streams_and_destroy():
    print("two optimizers on two streams", flush=True)
    a, b = Setup(SIZES, "bf16", "bf16", 8, seed=8), Setup(SIZES, "bf16", "bf16", 8, seed=9)
    streams = harness.Stream(), harness.Stream()
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=2)
    for s, st in zip((a, b), streams):
        s.opt.step(st.cuda_stream, seed=4, stochastic=True, **hyper)
    for s, st in zip((a, b), streams):
        st.synchronize()
        s.check(hyper, 1.0, 4)
        s.opt.destroy()


def test_the_moments_follow_differences_of_the_loss():
    """A quadratic loss: gradients by central differences in float64; a step with beta1 = beta2 = 0 moves every weight by lr in the
    gradient's direction (m / sqrt(v) is its sign) and a decaying one by lr weight_decay of itself more."""
    print("descent on a quadratic", flush=True)
    rng = np.random.default_rng(1)
    n = 500
    w, target = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n)

    def loss(x):
        return 0.5 * np.sum((x - target) ** 2)

    w64, h = w.astype(np.float64), 1e-4
    g = np.array([(loss(w64 + h * np.eye(1, n, k)[0]) - loss(w64 - h * np.eye(1, n, k)[0])) / (2 * h) for k in range(n)]).astype(np.float32)
    arena = Arena(n * 20 + 8192)
    t = dict(numel=n, grad=arena.add(g, 4, 0), master=arena.add(w, 4, 0), m=arena.add(np.zeros(n, np.float32), 4, 0), v=arena.add(np.zeros(n, np.float32), 4, 0), weight_decay=0.5)
    arena.upload()
    opt = B.Optimizer([t], grad_dtype=B.CKPT_F32, param_dtype=0)
    opt.step(0, step=1, lr=1e-3, beta1=0.0, beta2=0.0, eps=1e-12)
    harness.synchronize()
    arena.fetch()
    got = arena.read(1).view(np.float32).astype(np.float64)
    assert np.all(np.abs(got - (w64 * (1 - 5e-4) - 1e-3 * np.sign(g))) <= 2.0 ** -22 * (np.abs(w64) + 1e-3))
    assert loss(got) < loss(w64)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-8, 1e-12, 0.99e-12, 1e-15, 1e-20, 1e-25])
def test_second_moments_below_the_normal_numbers(bits, eps):
    """The root of a subnormal number counts where eps is as small; both sides of the rule that chooses how it is taken. The bound: as in check()."""
    print(f"adamw, subnormal second moments, eps {eps}, {bits} bits", flush=True)
    rng = np.random.default_rng(5)
    n = 4096 + 700
    v = (10.0 ** rng.uniform(-44, -36, n)).astype(np.float32)
    m = (rng.standard_normal(n) * np.sqrt(v.astype(np.float64))).astype(np.float32)
    w, g = np.zeros(n, np.float32), np.zeros(n, np.float32)
    arena = Arena(n * 20 + 16384)
    t = dict(numel=n, weight_decay=0.0, grad=arena.add(g, 4, 0), master=arena.add(w, 4, 0))
    if bits == 32:
        t |= dict(m=arena.add(m, 4, 0), v=arena.add(v, 4, 0))
    else:
        for name, x in (("m", m), ("v", v)):
            c, b = to.moment8(x, nonzero=name == "v")
            t |= {name: arena.add(c, 1, 0), name + "_scale": arena.add(b, 1, 0)}
            x[:] = to.values(c.reshape(1, -1), b.reshape(1, -1), to.MXFP8).reshape(-1)
    arena.upload()
    opt = B.Optimizer([t], grad_dtype=B.CKPT_F32, param_dtype=0, state_bits=bits)
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=eps, step=7)
    opt.step(0, **hyper)
    harness.synchronize()
    arena.fetch()
    m, v = to.moments(m, v, g, 1.0, 0.9, 0.95)
    assert np.count_nonzero((v > 0) & (v < 2.0 ** -126)) > 500
    want, update = to.adamw(w, m, v, weight_decay=0.0, **hyper)
    assert np.all(np.abs(arena.read(1).view(np.float32) - want) <= 2.0 ** -19 * np.abs(update) + 1e-38)


def test_a_nonfinite_gradient_without_the_norm_spoils_its_block_alone():
    print("infinity in a block", flush=True)
    s = Setup([1000], "f32", "bf16", 8, seed=12)
    at, _ = s.arena.parts[s.state[0]["index"]["grad"]]
    x = np.array([np.inf], np.float32)
    B.proxy_copy_h2d(s.arena.buf.ptr + at + 4 * 70, x.ctypes.data, 4)
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=3)
    s.opt.step(0, **hyper)
    harness.synchronize()
    s.arena.fetch()
    bad = np.zeros(32, bool)
    bad[70 // 32] = True
    for name in ("m", "v"):
        assert np.array_equal(s.part(0, name + "_scale") == 255, bad)
    w = s.part(0, "master").view(np.float32)
    assert np.isnan(w[70]) and np.isfinite(np.delete(w, 70)).all()


def test_offsets_beyond_32_bits():
    """One tensor of 2^32 + 1000 elements with 8-bit moments, 34 GB, zeros but for its end: gradient, weights and moments there change, nothing else does."""
    print("adamw of 4.3 G elements", flush=True)
    n, tail = (1 << 32) + 1000, 1500
    rng = np.random.default_rng(2)
    g, w = as_grad(1e-3 * rng.standard_normal(tail), "bf16"), (0.02 * rng.standard_normal(tail)).astype(np.float32)
    first = (n - tail) // 32 * 32
    g, w = np.concatenate([np.zeros(n - tail - first, g.dtype), g]), np.concatenate([np.zeros(n - tail - first, w.dtype), w])
    bufs = {"grad": harness.DevBuf(2 * n), "master": harness.DevBuf(4 * n), "m": harness.DevBuf(n), "v": harness.DevBuf(n),
            "m_scale": harness.DevBuf(-(-n // 32)), "v_scale": harness.DevBuf(-(-n // 32))}
    for b in bufs.values():
        B.proxy_device_fill_async(b.ptr, 0, b.nbytes, 0)
    B.proxy_copy_h2d(bufs["grad"].ptr + 2 * first, g.ctypes.data, g.nbytes)
    B.proxy_copy_h2d(bufs["master"].ptr + 4 * first, w.ctypes.data, w.nbytes)
    opt = B.Optimizer([dict(numel=n, weight_decay=0.1, **{k: b.ptr for k, b in bufs.items()})], grad_dtype=B.CKPT_BF16, param_dtype=0, state_bits=8)
    norm = harness.DevBuf(24)
    opt.grad_norm(norm.ptr, 0)
    opt.step(0, step=1, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, seed=3, stochastic=True, norm=norm.ptr)
    harness.synchronize()
    values = grad_values(g, "bf16")
    total = float(np.sum(values.astype(np.float64) ** 2))
    assert abs(B.ckpt_norm_result.from_buffer_copy(gu.download(norm).tobytes()).sum_squares - total) <= 1e-12 * total
    m, v = to.moments(np.zeros_like(w), np.zeros_like(w), values, 1.0, 0.9, 0.95)
    rm, rv = to.step_bits16(3, 1, first // 32, w.size)
    for name, x, r in (("m", m, rm), ("v", v, rv)):
        c, b = to.moment8(x, r, nonzero=name == "v")
        assert np.array_equal(gu.download(bufs[name], first, w.size), c) and np.array_equal(gu.download(bufs[name + "_scale"], first // 32, b.size), b)
        assert not gu.download(bufs[name], first - (1 << 20), 1 << 20).any()
    want, update = to.adamw(w, m, v, 1e-3, 0.9, 0.95, 1e-8, 1, 0.1)
    got = gu.download(bufs["master"], 4 * first, 4 * w.size).view(np.float32)
    assert np.all(np.abs(got - want) <= 2.0 ** -22 * np.abs(w) + 2.0 ** -19 * update + 1e-38)
    assert not gu.download(bufs["master"], 0, 1 << 20).any()
    opt.destroy()
    for b in bufs.values():
        b.free()


def test_what_is_refused():
    print("refusals", flush=True)
    buf, small = harness.DevBuf(1 << 16), harness.DevBuf(64)
    good = dict(numel=64, grad=buf.ptr, param=buf.ptr + 1024, master=buf.ptr + 2048, m=buf.ptr + 4096, v=buf.ptr + 8192, m_scale=buf.ptr + 12288, v_scale=buf.ptr + 12800, weight_decay=0.1)

    def refused(text, cfg=None, code=B.CKPT_EINVAL, **change):
        with pytest.raises(B.CkptError) as e:
            B.Optimizer([{**good, **change}], **{**dict(grad_dtype=B.CKPT_F32, state_bits=8), **(cfg or {})})
        assert e.value.code == code and text in e.value.text, e.value.text

    refused("grad_dtype", cfg=dict(grad_dtype=B.CKPT_I32))
    refused("param_dtype", cfg=dict(param_dtype=B.CKPT_F32))
    refused("state_bits", cfg=dict(state_bits=16))
    refused("dev_grad: null", grad=None)
    refused("dev_m: null", m=None)
    refused("dev_v_scale: null", v_scale=None)
    refused("dev_master: not aligned", master=buf.ptr + 2049)
    refused("dev_grad: not device memory", grad=good["grad"] * 0 + np.zeros(64, np.float32).ctypes.data)
    refused("dev_grad: range runs past", grad=small.ptr)
    refused("weight_decay", weight_decay=float("nan"))
    refused("too large", numel=1 << 60)
    with pytest.raises(B.CkptError):
        B.Optimizer([])
    with pytest.raises(B.CkptError):
        B.Optimizer([good, dict(numel=4, grad=buf.ptr)], grad_dtype=B.CKPT_F32, state_bits=8)
    opt = B.Optimizer([good], grad_dtype=B.CKPT_F32, state_bits=8)
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(lr=float("inf")), dict(norm=buf.ptr + 4), dict(norm=small.ptr + 48)):
        with pytest.raises(B.CkptError) as e:
            opt.step(0, **{**dict(step=1, lr=1e-3), **bad})
        assert e.value.code == B.CKPT_EINVAL
    for bad in (dict(out=None), dict(out=buf.ptr + 4), dict(out=buf.ptr, max_norm=float("nan")), dict(out=buf.ptr, grad_scale=float("inf"))):
        with pytest.raises(B.CkptError) as e:
            opt.grad_norm(stream=0, **bad)
        assert e.value.code == B.CKPT_EINVAL
    harness.synchronize()


def test_a_negative_grad_scale_is_refused():
    """It would make the norm negative, and nothing would be clipped."""
    print("negative grad_scale", flush=True)
    buf = harness.DevBuf(4096)
    opt = B.Optimizer([dict(numel=64, grad=buf.ptr)], grad_dtype=B.CKPT_F32)
    with pytest.raises(B.CkptError) as e:
        opt.grad_norm(buf.ptr + 1024, 0, max_norm=1.0, grad_scale=-1.0)
    assert e.value.code == B.CKPT_EINVAL
