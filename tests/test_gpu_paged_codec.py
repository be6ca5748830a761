"""The paged calls and the codec as a serving program uses them together: prompts of two sequences in uneven chunks
(append, attention), the finished prompt out of the pages into varrate_encode, then new tokens decoded on the coded
cache with the exact tail out of the pages, beside attention over the pages themselves."""
import math

import pytest
import torch

from gpu_helpers import V, decode_close, f64
from paged_helpers import D, DT, HALF, close, form

pytestmark = pytest.mark.gpu

L, G, GRP, N, W, PS, STEPS = 2, 2, 4, 211, 8, 32, 4
H = G * GRP
EPS = 1e-6
CHUNKS = [(80, 50), (0, 3), (100, 157), (31, 1)]     # new tokens of the two sequences


@pytest.fixture(scope="module", autouse=True)
def _gpu(vlib):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


class Program:
    def __init__(self, dtype):
        self.dtype, self.dt = dtype, DT[dtype]
        self.gen = torch.Generator().manual_seed(11)
        per = -(-(N + STEPS) // PS)
        self.pages = V.PagedCache.allocate(L, 2 * per + 2, G, PS, V.BF16 if dtype == "bf16" else V.F32)
        self.pages.pool.fill_(float("nan"))
        order = torch.randperm(2 * per + 2, generator=self.gen)[:2 * per].reshape(2, per)
        self.table_host, self.table = order, order.to(torch.int32).cuda()
        self.len, self.status = [0, 0], torch.zeros(1, dtype=torch.int32, device="cuda")
        self.freq = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
        self.wq, self.wk = ((1 + 0.2 * torch.randn(D, generator=self.gen)).to(self.dt).cuda() for _ in range(2))
        self.queries = [[[] for _ in range(L)] for _ in range(2)]

    def seqs(self, new):
        start = [0, new[0], sum(new)]
        return V.SeqBatch.of(torch.tensor(start, dtype=torch.int32, device="cuda"),
                             torch.tensor(self.len, dtype=torch.int32, device="cuda"), self.table, sum(new))

    def tokens(self, s, c, layer, lo, hi):
        u = torch.arange(lo, hi)
        page = self.table_host[s][u // PS].cuda()
        return self.pages.pool[layer, page, c, :, (u % PS).cuda()].double().transpose(0, 1)     # [G][tokens][d]

    def take(self, new):
        """A chunk of new tokens through every layer: appended, attended to; both against 64 bits. Queries and outputs."""
        self.len = [a + b for a, b in zip(self.len, new)]
        seqs, T = self.seqs(new), sum(new)
        ws = V.paged_attn_workspace(self.pages, seqs, GRP)
        outs = []
        for layer in range(L):
            x = torch.randn((T, (H + 2 * G) * D), generator=self.gen).to(self.dt).cuda()
            q, k, v = (y.unflatten(1, (-1, D)) for y in x.split((H * D, G * D, G * D), dim=1))
            q_out = torch.empty((T, H, D), dtype=self.dt, device="cuda")
            out = torch.empty_like(q_out)
            V.check(V.varrate_paged_append(self.pages, seqs, layer, q, k, v, self.wq, self.wk, EPS, self.freq, D, q_out, self.status))
            V.check(V.varrate_paged_attn(self.pages, seqs, layer, GRP, q_out, out, self.status, ws))
            outs.append((q_out, out))
            for s in range(2):
                lo, hi, n, total = sum(new[:s]), sum(new[:s + 1]), new[s], self.len[s]
                pos = torch.arange(total - n, total, device="cuda")
                fp32 = 32 * 2.0 ** -24
                for got, src, w in ((q_out[lo:hi], q[lo:hi], self.wq), (self.tokens(s, 0, layer, total - n, total).transpose(0, 1), k[lo:hi], self.wk)):
                    want, size = form(src, w, EPS, self.freq, D, pos)
                    close(got, want, fp32 * size + HALF[self.dtype] * (want.abs() + fp32 * size))
                assert torch.equal(self.tokens(s, 1, layer, total - n, total).transpose(0, 1), v[lo:hi].double())
                kk, vv = self.tokens(s, 0, layer, 0, total), self.tokens(s, 1, layer, 0, total)
                seen = torch.arange(total, device="cuda")[None] <= pos[:, None]
                for h in range(H):
                    g = h // GRP
                    qd = q_out[lo:hi, h].double()
                    a = torch.softmax((qd @ kk[g].T / math.sqrt(D)).masked_fill(~seen, -math.inf), -1)
                    want, mass = a @ vv[g], a @ vv[g].abs()
                    ds = 132 * 2.0 ** -23 * (qd.abs() @ kk[g].abs().T / math.sqrt(D)).amax(-1, keepdim=True) if n else 0
                    rel = 2 * ds + 2.0 ** -20 + 2 * (total + 8) * 2.0 ** -24 + (2.0 ** -8 if self.dtype == "bf16" else 0)
                    close(out[lo:hi, h], want, rel * mass + HALF[self.dtype] * (want.abs() + rel * mass))
                self.queries[s][layer].append(q_out[lo:hi].clone())
        return outs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_from_prompt_chunks_to_decode_on_the_codec(dtype):
    p = Program(dtype)
    for new in CHUNKS:
        p.take(new)
    assert p.len == [N, N]
    seqs = p.seqs((0, 0))
    k, v = (torch.full((2, L, G, N, D), float("nan"), dtype=p.dt, device="cuda") for _ in range(2))
    V.check(V.varrate_paged_gather(p.pages, seqs, 0, L, None, N, k, v, p.status))
    for s in range(2):
        for l in range(L):
            assert torch.equal(k[s, l].double(), p.tokens(s, 0, l, 0, N)) and torch.equal(v[s, l].double(), p.tokens(s, 1, l, 0, N))
    # the whole cache kept (budget 1): every token at full rank, so that decode is attention up to the coded values' rounding
    cfg = V.make_config(L, G, GRP, N, batch=2, budget_frac=1.0, r_min=16, window=W, dtype=V.BF16 if dtype == "bf16" else V.F32)
    q_win = torch.stack([torch.stack([torch.cat(p.queries[s][l])[-W:] for l in range(L)]) for s in range(2)])
    basis = torch.linalg.qr(torch.randn((2, L, G, D, D), generator=p.gen, dtype=torch.float64))[0].to(p.dt).cuda().contiguous()
    packed = V.PackedCache.allocate(cfg)
    V.check(V.varrate_encode(cfg, q_win.contiguous(), k, v, basis[0], basis[1], None, packed, None, p.status, V.workspace(cfg, V.CALL_ENCODE)))
    ws = V.workspace(cfg, V.CALL_DECODE)
    first = torch.full((2,), N, dtype=torch.int32, device="cuda")
    for step in range(1, STEPS + 1):
        outs = p.take((1, 1))
        for l in range(L):
            tail = [torch.empty((2, 1, G, step, D), dtype=p.dt, device="cuda") for _ in range(2)]
            V.check(V.varrate_paged_gather(p.pages, p.seqs((1, 1)), l, 1, first, step, *tail, p.status))
            q, exact = outs[l]
            out = torch.empty_like(q)
            V.check(V.varrate_decode_attn(cfg, packed, basis[0], basis[1], q, l, tail[0], tail[1], step, out, p.status, ws))
            for s in range(2):
                kk, vv = p.tokens(s, 0, l, 0, N + step), p.tokens(s, 1, l, 0, N + step)
                want = torch.stack([torch.softmax(q[s, h].double() @ kk[h // GRP].T / math.sqrt(D), -1) @ vv[h // GRP] for h in range(H)])
                assert decode_close(f64(out[s]), f64(want), cfg)
                assert decode_close(f64(out[s]), f64(exact[s]), cfg)
    torch.cuda.synchronize()
    assert int(p.status.item()) == V.OK
