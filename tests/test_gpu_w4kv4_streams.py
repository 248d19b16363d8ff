"""The 4-bit operators' torch calls run on torch's current stream."""
import numpy as np
import pytest

import synth
import w4kv4_ref as ref

pytestmark = pytest.mark.gpu


class _Step:
    """The attention half of a decoder block in 4 bits, as the README writes it: no
    call names a stream."""

    def __init__(self, B=2, d=256, H=4, Hkv=2, dh=64, cap=64, past=20):
        import torch
        from paper_2608_14586_amd import binding as vb
        self.B, self.d, self.H, self.Hkv, self.dh, self.cap = B, d, H, Hkv, dh, cap
        rng = np.random.default_rng(synth.seed_of("streams"))
        self.N = (H + 2 * Hkv) * dh

        def packed(N, K):
            codes = torch.from_numpy(rng.integers(0, 16, (N, K), dtype=np.uint8)).cuda()
            s = ref.to_dev(rng.uniform(0.002, 0.01, (N, K // 128)))
            Wp = torch.empty(vb.vla_op_w4_packed_bytes(N, K, 128), dtype=torch.uint8, device="cuda")
            vb.vla_op_w4_pack(codes, s, None, Wp, 128)
            return Wp

        self.Wqkv, self.Wo = packed(self.N, d), packed(d, H * dh)
        ang = np.arange(cap)[:, None] * 10000.0 ** (-np.arange(0, dh, 2) / dh)
        self.cos, self.sin = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))
        self.g = torch.ones(dh, device="cuda")
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.x, self.qkv, self.q, self.k, self.o = bf(B, d), bf(B, self.N), bf(B, 1, H, dh), bf(B, 1, Hkv, dh), bf(B, 1, H, dh)
        self.h = torch.zeros((B, d), device="cuda")
        self.pos = torch.full((B, 1), past, dtype=torch.int32, device="cuda")
        self.lens = torch.full((B,), past + 1, dtype=torch.int32, device="cuda")
        self.cache = torch.zeros(vb.vla_op_kv4_bytes(B, Hkv, cap, dh), dtype=torch.uint8, device="cuda")
        rows = ref.to_dev(ref.normal(("streamsrows",), (B, past, Hkv, dh)))
        vb.vla_op_kv4_store(rows, rows, None, None, self.cache, cap)
        n = vb.vla_op_attention_kv4_scratch(B, 1, H, Hkv, dh, cap)
        self.scratch = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        self.back = bf(B, 1, Hkv, dh), bf(B, 1, Hkv, dh)
        torch.cuda.synchronize()

    def run(self, x):
        from paper_2608_14586_amd import binding as vb
        self.x.copy_(x)  # on the current stream, as all that follows
        self.h.fill_(0.5)
        vb.vla_op_gemv_w4(self.x, self.Wqkv, None, self.qkv, self.N, 128)
        rows = self.qkv.view(self.B, 1, self.H + 2 * self.Hkv, self.dh)
        vb.vla_op_qk_norm_rope(rows[:, :, :self.H], rows[:, :, self.H:self.H + self.Hkv], self.g, self.g, 1e-6, self.cos, self.sin,
                               self.pos, self.q, self.k)
        vb.vla_op_kv4_store(self.k, rows[:, :, self.H + self.Hkv:], self.pos.view(-1), None, self.cache, self.cap)
        vb.vla_op_kv4_load(self.cache, self.cap, self.pos.view(-1), None, *self.back)
        vb.vla_op_attention_kv4(self.q, self.cache, self.cap, self.Hkv, self.lens, self.o, self.cap, 0, 0, self.scratch)
        vb.vla_op_gemv_w4(self.o.view(self.B, -1), self.Wo, self.h, self.h, self.d, 128)

    def results(self):
        return [t.clone() for t in (self.h, self.q, self.k, self.cache) + self.back]


def _inputs(i):
    return ref.to_dev(ref.normal(("streamsx", i), (2, 256)))


def _equal(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_the_step_without_a_stream_can_be_captured():
    import torch
    s = _Step()
    x = _inputs(0)
    s.run(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run(x)
    for i in range(4):
        x.copy_(_inputs(i))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = s.results()
        s.run(x)  # eagerly
        assert _equal(got, s.results()), i


def test_calls_follow_their_inputs_on_a_side_stream():
    """Inputs that a side stream makes behind long work of its own: the calls wait for them."""
    import torch
    s = _Step()
    want = []
    for i in range(3):
        s.run(_inputs(i))
        want.append(s.results())
    xs = [_inputs(i) for i in range(3)]
    a = torch.ones((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for i in range(3):
        with torch.cuda.stream(side):
            b = a
            for _ in range(8):
                b = (b @ a) * (1 / 4096)
            s.run(xs[i] * b[0, 0])  # times 1
            got = s.results()
        side.synchronize()
        assert _equal(got, want[i]), i


def test_packing_on_a_side_stream():
    import torch
    from paper_2608_14586_amd import binding as vb
    codes = torch.randint(0, 16, (64, 256), dtype=torch.uint8, device="cuda")
    scales = torch.rand((64, 2), device="cuda").bfloat16()
    want = torch.zeros(vb.vla_op_w4_packed_bytes(64, 256, 128), dtype=torch.uint8, device="cuda")
    vb.vla_op_w4_pack(codes, scales, None, want, 128)
    a, late, got = torch.ones((4096, 4096), device="cuda"), torch.zeros_like(codes), torch.zeros_like(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(8):
            a = (a @ a) * (1 / 4096)
        late.copy_(codes * (a[0, 0] > 0))
        vb.vla_op_w4_pack(late, scales, None, got, 128)
    side.synchronize()
    assert torch.equal(got, want)


def test_a_stream_by_its_address():
    """0 is the null stream, whatever the current one."""
    import torch
    from paper_2608_14586_amd import binding as vb
    s = _Step()
    x = _inputs(1)
    y, z = torch.zeros_like(s.qkv), torch.zeros_like(s.qkv)
    vb.vla_op_gemv_w4(x, s.Wqkv, None, y, s.N, 128)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        vb.vla_op_gemv_w4(x, s.Wqkv, None, z, s.N, 128, stream=0)
    torch.cuda.default_stream().synchronize()
    assert torch.equal(y, z)
