"""Edges of the paged calls on the GPU: headers of the workspace that a call may find, values as large and as small as their
type holds, norms of zeros, row ranges out of order, rows without a finite score, every number of heads in a group. Tolerances
are derived in paged_helpers."""
import pytest
import torch

from paged_helpers import D, V, Batch, attn_ref, close
from test_gpu_paged import NAN, run_attn, status

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu(vlib):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


# ------------------------------------------------------------------------------------ the header of the workspace

def ctas(dtype):
    return torch.cuda.get_device_properties(0).multi_processor_count * (1 if dtype == "bf16" else 2)


def found(b, ws, headers):
    """A call that finds such words at the start of the workspace raises CORRUPT; the call after it is right."""
    q = b.rows(b.H)
    want, tol = attn_ref(b, q)
    for words in headers:
        ws[:4 * len(words)].view(torch.int32).copy_(torch.tensor(words, dtype=torch.int32))
        for expected in (V.ERR_CORRUPT, V.OK):
            b.status.zero_()
            out = torch.full_like(q, NAN)
            assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, ws) == V.OK
            assert status(b) == expected
        close(out, want, tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_counter_found_used_with_units_left_to_take(dtype):
    """More units than CTAs (one key tile a sequence, so a unit is a sequence and a head): a count that is not zero takes units
    away without the counter's end showing it."""
    units, C = 1000, ctas(dtype)
    assert C < units
    b = Batch([(1, s % 30) for s in range(units // 2)], dtype, 2, 4)
    found(b, b.workspace(), [[c] for c in (1, 3, units - C - 1, units - C, units - C + 1, units - 1, units)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_counter_found_used_by_a_long_prompt(dtype):
    b = Batch([(3000, 100), (1, 2000)], dtype, 4, 2)
    found(b, b.workspace(), [[1], [3], [100]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_header_never_zeroed(dtype):
    """Every word of the header holds something, as a call whose merge was never launched leaves it."""
    b = Batch([(1, s % 30) for s in range(500)], dtype, 2, 4)
    found(b, b.workspace(), [[c, 0, 1, 1000, 0, 1000, 1, 1] for c in (0, 1, 3, 100, 1000)])


# ------------------------------------------------------------------------------------ values at the ends of their type

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [124, -90])
@pytest.mark.parametrize("lens", [[(1, 2000), (1, 7)], [(150, 600), (1, 900)], [(1, 9999)], [(40, 5000)]], ids=str)
def test_attn_values_near_the_ends_of_the_range(dtype, power, lens):
    """A mean of values is no larger than the largest one, however many keys there are and however far scores rise: values
    of 2^126 give finite results, values of 2^-90 keep their precision."""
    b = Batch(lens, dtype, 1, 8, 64)
    b.pool[:, :, 1] *= 2.0 ** power
    run_attn(b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("jump", [10.0, 16.0, 17.0, 25.0, 60.0, 100.0])
@pytest.mark.parametrize("lens", [[(1, 400)], [(130, 271)]], ids=str)
def test_attn_large_values_and_a_score_that_rises(dtype, jump, lens):
    """The keys from some position on stand `jump` above the ones before."""
    for at in (20, 40, 100, 130, 300):
        b = Batch(lens, dtype, 1, 4)
        b.pool[:, :, 1] *= 2.0 ** 124
        q = b.rows(b.H)
        q[..., 0] = 16.0
        for u in range(b.len[0]):
            b.pool[0, b.table_host[0, u // b.ps], 0, 0, u % b.ps, 0] = jump * D ** 0.5 / 16.0 if u >= at else 0.0
        run_attn(b, q=q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_large_values_of_one_sign_and_equal_scores(dtype):
    """The sum of the weights reaches the number of keys: as many times the values must not appear on the way."""
    b = Batch([(1, 20000), (200, 3000)], dtype, 1, 2, 128)
    b.pool[:, :, 1] = b.pool[:, :, 1].abs() * 2.0 ** 124
    run_attn(b, q=torch.zeros((b.T, b.H, D), dtype=b.dt, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_scores_that_rise_slowly(dtype):
    """Every key stands a little above the one before it: the sum of the weights comes near its bound again and again."""
    b = Batch([(1, 6000), (140, 1500)], dtype, 1, 4, 64)
    q = b.rows(b.H)
    q[..., 0] = 16.0
    for s in range(2):
        for u in range(b.len[s]):
            b.pool[0, b.table_host[s, u // b.ps], 0, 0, u % b.ps, 0] = u * (0.25 if s else 0.0625) * D ** 0.5 / 16.0
    b.pool[:, :, 1] *= 2.0 ** 124
    run_attn(b, q=q)


# ------------------------------------------------------------------------------------ norms

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [1e-45, 1e-46, 1e-300, 1e-6])
def test_append_norm_of_zeros(dtype, eps):
    """A head of zeros is zeros after its norm wherever eps is above zero, one that fp32 cannot hold included."""
    b = Batch([(5, 3)], dtype, 2, 2)
    q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
    q[1], k[2], q[3, 1] = 0.0, 0.0, 0.0
    w = torch.ones(D, dtype=b.dt, device="cuda")
    q_out = torch.full_like(q, NAN)
    assert V.varrate_paged_append(b.pages, b.seqs, 0, q, k, v, w, w, eps, None, 0, q_out, b.status) == V.OK
    assert (q_out[1] == 0).all() and (q_out[3, 1] == 0).all() and (b.tokens(0, 0)[:, 3 + 2] == 0).all()
    assert torch.isfinite(q_out).all() and torch.isfinite(b.tokens(0, 0)).all()
    assert status(b) == V.OK


# ------------------------------------------------------------------------------------ row ranges out of order

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("start", [[4, 8, 0, 4], [9, 5, 3, 0], [0, 9, 2, 9], [8, 2, 9, 9]], ids=str)
def test_row_ranges_out_of_order(dtype, start):
    """Reported, and nothing outside the rows and the sequences' own places in the pages is written."""
    b = Batch([(3, 30), (3, 40), (3, 50)], dtype, 2, 2)
    b.row_start.copy_(torch.tensor(start, dtype=torch.int32))
    q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
    own = torch.zeros(b.pool.shape, dtype=torch.bool, device="cuda")
    for s in range(3):
        for u in range(b.len[s]):
            own[0, b.table_host[s, u // b.ps], :, :, u % b.ps] = True
    rest = b.pool.clone()
    big = torch.full((b.T + 2, b.H, D), 7.0, dtype=b.dt, device="cuda")
    assert V.varrate_paged_append(b.pages, b.seqs, 0, q, k, v, None, None, 0.0, None, 0, big[1:-1], b.status) == V.OK
    assert status(b) == V.ERR_CORRUPT
    assert (big[0] == 7).all() and (big[-1] == 7).all()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(b.pool.view(bits)[~own], rest.view(bits)[~own])
    b.status.zero_()
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, big[1:-1], b.status, b.workspace()) == V.OK
    assert status(b) == V.ERR_CORRUPT
    assert (big[0] == 7).all() and (big[-1] == 7).all()


# ------------------------------------------------------------------------------------ rows without a finite score

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grp", [1, 4, 7])
@pytest.mark.parametrize("lens", [[(1, 0)], [(1, 700), (1, 3)], [(150, 300)], [(300, 0), (1, 1000)], [(1, 9999)]], ids=str)
def test_attn_scores_of_minus_infinity(dtype, grp, lens):
    """Keys whose score is -infinity for some queries: rows that see nothing else give zeros, the others leave them out."""
    b = Batch(lens, dtype, 2, grp, 64)
    q = b.rows(b.H)
    q[..., 0] = q[..., 0].abs() + 0.5
    finite = [0, 200]                        # KV head 0: no key; KV head 1: the keys from position 200 on, then every third
    for s in range(len(lens)):
        for u in range(b.len[s]):
            at = (b.table_host[s, u // b.ps], u % b.ps)
            b.pool[0, at[0], 0, 0, at[1], 0] = -float("inf")
            if u < finite[1] or u % 3:
                b.pool[0, at[0], 0, 1, at[1], 0] = -float("inf")
    want, tol = attn_ref(b, q)
    for s, (n, c) in enumerate(lens):
        rows = torch.arange(b.start[s], b.start[s + 1], device="cuda")
        seen = torch.arange(c, c + n, device="cuda")
        want[rows, :grp] = 0.0
        tol[rows, :grp] = 0.0
        none = rows[seen < 201]              # 201 is the first multiple of three from 200 on
        want[none, grp:] = 0.0
        tol[none, grp:] = 0.0
    assert not torch.isnan(want).any()
    out = torch.full((b.T, b.H, D), NAN, dtype=b.dt, device="cuda")
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, b.workspace()) == V.OK
    close(out, want, tol)
    assert status(b) == V.OK


# ------------------------------------------------------------------------------------ heads of a group

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grp", [2, 3, 5, 6])
@pytest.mark.parametrize("lens", [[(1, 0)], [(1, 700), (1, 3), (1, 129)], [(64, 64), (0, 5), (3, 200)], [(129, 0)],
                                  [(300, 0), (1, 1000), (33, 95)], [(40, 1500)]], ids=str)
def test_attn_heads_of_a_group(dtype, grp, lens):
    """Groups whose query tiles leave rows of the matrix product unused (126 or 125 of 128) among them."""
    run_attn(Batch(lens, dtype, 2, grp, pad=2, lead=1))
