"""The four-bit key/value cache and attention over it, on the GPU through the C ABI against plain implementations in 64 bits (kv_reference.py): codes, scales and
values read back exactly, attention within what 32-bit sums and weights of 11 bits allow."""
import random

import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2409_17870_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.load()
    return torch, binding


class Batch:
    """A cache of random contents, a batch of sequences whose pages lie scattered in it, and new rows of q, k and v."""

    def __init__(self, torch, dtype, D, heads, groups, ps, lengths, new, seed=1, spare=2, fused=True, room=0):
        g = torch.Generator().manual_seed(seed)
        r = random.Random(seed)
        pages_of = [-(-n // ps) for n in lengths]
        pages, width = sum(pages_of) + spare, max(1, max(pages_of)) + room
        order = r.sample(range(pages), sum(pages_of))
        self.table = torch.full((len(lengths), width), -1, dtype=torch.int32)
        for b, n in enumerate(pages_of):
            self.table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
        self.lengths, self.starts = list(lengths), [0]
        for n in new:
            self.starts.append(self.starts[-1] + n)
        self.tokens, self.dtype = self.starts[-1], dtype

        def rows(*shape):
            x = torch.randn(shape, generator=g)
            x[..., 3::29] *= 4.0
            return (x * torch.exp(0.4 * torch.randn(shape[:-1] + (1,), generator=g))).to(dtype)
        self.hk, self.hv = rows(pages, heads, ps, D), rows(pages, heads, ps, D)
        (uk, sk), (uv, sv) = ref.quantise(self.hk), ref.quantise(self.hv)
        self.codes, self.scales = ref.layout(uk, uv).cuda(), torch.stack([sk, sv], 2).cuda().contiguous()
        if fused:
            x = rows(self.tokens, heads * groups + 2 * heads, D).cuda()
            self.q, self.k, self.v = x[:, :heads * groups], x[:, heads * groups:heads * groups + heads], x[:, heads * groups + heads:]
        else:
            self.q, self.k, self.v = (rows(self.tokens, n, D).cuda() for n in (heads * groups, heads, heads))
        self.args = [self.codes, self.scales, self.table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()]
        self.starts_gpu = torch.tensor(self.starts, dtype=torch.int32).cuda()

    def attention(self, q, window, sinks, scale):
        return ref.attention(q, self.codes, self.scales, self.table, self.lengths, self.starts, window, sinks, scale)


def close(torch, got, want, near):
    half = 2.0 ** (-11 if got.dtype == torch.float16 else -8)  # half a unit of the last place of its type, relative
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 0.0
    d = (got.cpu().double() - want).abs()
    bad = d > near + half * (want.abs() + near) + tiny
    assert not bool(bad.any()), "%d of %d off, worst %.3g allowed %.3g" % (int(bad.sum()), bad.numel(), float(d[bad].max()), float(near[bad].min()))


# ------------------------------------------------------------------ store ---
STORES = [  # D, heads, page, lengths, new
    (128, 1, 16, [1], [1]),
    (128, 32, 16, [777], [1]),
    (64, 3, 16, [9, 8, 7, 16, 17, 33], [9, 1, 7, 16, 2, 20]),
    (128, 5, 64, [130, 64, 1, 0, 200], [130, 3, 1, 2, 17]),          # one sequence without a place for its two tokens
    (64, 8, 32, [100] * 70, [1] * 70),                               # more sequences than lanes
    (128, 2, 256, [300, 300], [44, 300]),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("case", range(len(STORES)))
def test_write_and_read_are_exact(gpu, dtype, case):
    torch, binding = gpu
    D, heads, ps, lengths, new = STORES[case]
    dt = getattr(torch, dtype)
    x = Batch(torch, dt, D, heads, 2, ps, lengths, new, seed=case)
    before_codes, before_scales = ref.unlayout(x.codes, ps), x.scales.cpu().clone()
    binding.apmm_kv_write(x.k, x.v, *x.args, x.starts_gpu)
    after = ref.unlayout(x.codes, ps)
    want = [c.clone() for c in before_codes]
    want_scales = before_scales.clone()
    rk, rv = torch.zeros(x.k.shape, dtype=dt), torch.zeros(x.v.shape, dtype=dt)
    for i, rows in enumerate((x.k, x.v)):
        u, s = ref.quantise(rows.cpu())
        for b, length in enumerate(lengths):
            for t in range(new[b]):
                pos, row = length - new[b] + t, x.starts[b] + t
                if pos < 0:
                    continue
                page = int(x.table[b, pos // ps])
                want[i][page, :, pos % ps] = u[row]
                want_scales[page, :, i, pos % ps] = s[row]
                (rk, rv)[i][row] = ref.value(u[row], s[row])
    for i in range(2):
        assert torch.equal(after[i], want[i])
    assert torch.equal(x.scales.cpu(), want_scales)
    k, v = binding.apmm_kv_read(*x.args, x.tokens, x.starts_gpu)
    assert torch.equal(k.cpu(), rk) and torch.equal(v.cpu(), rv)


@pytest.mark.parametrize("heads", [32, 33])
def test_large_writes_and_reads_are_the_small_ones(gpu, heads):
    """Heads of 64 channels go two to a wave in large calls: the same cache and rows as from calls of one sequence."""
    torch, binding = gpu
    lengths, new = [1500, 777, 1800, 9], [1490, 777, 1793, 0]
    x = Batch(torch, torch.float16, 64, heads, 1, 16, lengths, new, seed=31)
    assert (sum(new) // 8 + 2 * len(new)) * heads >= 16384 > (max(new) // 8 + 2) * heads  # the eights that a call may touch, as the launch counts them
    large, small = [(x.codes.clone(), x.scales.clone()) for _ in range(2)]
    binding.apmm_kv_write(x.k, x.v, *large, *x.args[2:], x.starts_gpu)
    k, v = binding.apmm_kv_read(*large, *x.args[2:], x.tokens, x.starts_gpu)
    for b, n in enumerate(new):
        rows = slice(x.starts[b], x.starts[b + 1])
        one = (x.args[2][b:b + 1], x.args[3][b:b + 1])
        starts = torch.tensor([0, n], dtype=torch.int32).cuda()
        binding.apmm_kv_write(x.k[rows], x.v[rows], *small, *one, starts)
        k1, v1 = binding.apmm_kv_read(*small, *one, n, starts)
        assert torch.equal(k1, k[rows]) and torch.equal(v1, v[rows])
    assert torch.equal(large[0], small[0]) and torch.equal(large[1], small[1])


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_borders_of_the_grid(gpu, dtype):
    """Numbers on and beside the cells' borders, zeros, the smallest and the largest numbers, and rows that are not finite."""
    torch, binding = gpu
    dt = getattr(torch, dtype)
    D, n = 64, 40
    info = torch.finfo(dt)
    g = torch.Generator().manual_seed(3)
    x = torch.zeros((n, 1, D), dtype=dt)
    for r in range(16):  # even multiples of a scale that divides them, and their neighbours
        s = 2.0 ** (r - 8)
        grid = torch.tensor([(c - 16) * s for c in range(1, 32)], dtype=torch.float64).to(dt)
        x[r, 0, :31] = grid
        x[r, 0, 31:47] = torch.nextafter(grid[:16].float(), torch.tensor(0.0)).to(dt)
        x[r, 0, 47:62] = -grid[:15]
        x[r, 0, 0] = 15 * s
    x[16] = 0.0
    x[17] = -0.0
    x[18, 0, 5] = info.smallest_normal
    x[19, 0, 5] = info.smallest_normal * info.eps          # the smallest number there is
    x[20, 0, ::3] = info.smallest_normal * info.eps * 9
    x[21, 0, 0], x[21, 0, 1], x[21, 0, 2] = info.max, -info.max, 1.0
    x[22, 0, 7], x[23, 0, 7], x[24, 0, 7] = float("nan"), float("inf"), -float("inf")
    x[25, 0] = info.max
    x[26, 0, 0], x[26, 0, 1:] = 1.0, -info.smallest_normal * info.eps   # just below zero: the cell below
    x[27, 0, 0], x[27, 0, 1:] = -1.0, info.smallest_normal
    x[28:] = (torch.randn((n - 28, 1, D), generator=g) * info.smallest_normal * 3).to(dt)
    codes, scales = binding.apmm_kv_cache(3, 16, 1, D, dt)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda()
    lengths, starts = torch.tensor([n], dtype=torch.int32).cuda(), torch.tensor([0, n], dtype=torch.int32).cuda()
    binding.apmm_kv_write(x.cuda(), x.flip(0).contiguous().cuda(), codes, scales, table, lengths, starts)
    got = binding.apmm_kv_read(codes, scales, table, lengths, n, starts)
    for rows, back in ((x, got[0].cpu()), (x.flip(0), got[1].cpu())):
        want = ref.value(*ref.quantise(rows))
        assert torch.equal(torch.isnan(back), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(back, nan=7.0), torch.nan_to_num(want, nan=7.0))


@pytest.mark.parametrize("how", ["odd address", "odd stride", "heads first"])
def test_rows_at_any_address(gpu, how):
    torch, binding = gpu
    D, heads, new = 128, 4, [13, 1, 8]
    x = Batch(torch, torch.float16, D, heads, 3, 32, [40, 65, 8], new, seed=4, fused=False)

    def moved(t):
        if how == "odd address":
            flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape)
        elif how == "odd stride":
            flat = torch.empty((t.shape[0], t.shape[1] * (D + 1) + 3), dtype=t.dtype, device=t.device)[:, :t.shape[1] * (D + 1)].unflatten(1, (t.shape[1], D + 1))[:, :, :D]
        else:
            flat = torch.empty((t.shape[1], t.shape[0], t.shape[2]), dtype=t.dtype, device=t.device).transpose(0, 1)
        flat.copy_(t)
        return flat
    plain = [x.codes.clone(), x.scales.clone()]
    binding.apmm_kv_write(x.k, x.v, *plain, *x.args[2:], x.starts_gpu)
    binding.apmm_kv_write(moved(x.k), moved(x.v), *x.args, x.starts_gpu)
    assert torch.equal(plain[0], x.codes) and torch.equal(plain[1], x.scales)
    k, v = binding.apmm_kv_read(*x.args, x.tokens, x.starts_gpu)
    k2, v2 = moved(torch.zeros_like(k)), moved(torch.zeros_like(v))
    binding.apmm_kv_read(*x.args, x.tokens, x.starts_gpu, k_out=k2, v_out=v2)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    o = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu)
    o2 = moved(torch.zeros_like(o))
    binding.apmm_kv_attention(moved(x.q), *x.args, x.starts_gpu, out=o2)
    assert torch.equal(o, o2)


# -------------------------------------------------------------- attention ---
ATTENDS = [  # D, heads, groups, page, lengths, new, window, sinks
    (128, 1, 1, 16, [1], [1], 0, 0),
    (128, 2, 1, 16, [31, 32, 33, 1, 0, 64, 127, 250], [1] * 8, 0, 0),
    (64, 2, 8, 32, [5, 100, 257], [1] * 3, 0, 0),
    (128, 3, 3, 16, [300, 41], [2, 5], 0, 0),                        # 16 rows and fewer, queries of several tokens
    (64, 1, 40, 64, [70, 200], [1, 1], 0, 0),                        # more heads than rows of a workgroup
    (128, 2, 4, 16, [1500], [1], 0, 0),                              # cut in pieces
    (64, 1, 1, 128, [4000], [1], 0, 0),
    (128, 2, 2, 16, [200, 90, 33, 0], [1, 1, 1, 1], 50, 0),
    (64, 2, 2, 16, [200, 90, 33, 700], [1, 3, 1, 1], 1, 0),
    (128, 2, 2, 32, [200, 90, 33, 700], [1, 1, 2, 1], 40, 5),
    (64, 2, 1, 16, [300], [1], 3, 100),
    (128, 1, 1, 16, [200], [200], 0, 0),                             # prompts
    (64, 2, 2, 32, [130, 77, 1], [130, 77, 1], 0, 0),
    (128, 2, 3, 64, [300, 50], [111, 50], 0, 0),
    (64, 1, 4, 16, [333], [150], 60, 0),
    (128, 1, 2, 16, [333, 40], [150, 40], 60, 37),
    (128, 2, 1, 16, [40, 3], [50, 9], 0, 0),                         # more new tokens than the lengths say: the first see nothing
    (64, 1, 1, 16, [900], [100], 0, 0),                              # a prompt's last piece, cut in pieces
    (128, 1, 5, 32, [600, 17, 0, 290], [60, 1, 1, 290], 100, 10),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("case", range(len(ATTENDS)))
def test_attention(gpu, dtype, case):
    torch, binding = gpu
    D, heads, groups, ps, lengths, new, window, sinks = ATTENDS[case]
    x = Batch(torch, getattr(torch, dtype), D, heads, groups, ps, lengths, new, seed=case)
    got = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu, window=window, sinks=sinks)
    close(torch, got, *x.attention(x.q, window, sinks, D ** -0.5))
    if all(n == 1 for n in new):
        assert torch.equal(got, binding.apmm_kv_attention(x.q, *x.args, window=window, sinks=sinks))
    assert torch.equal(got, binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu, window=window, sinks=sinks))  # no order that changes


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("new", [1, 90])
def test_large_and_small_numbers(gpu, dtype, new):
    """Queries and scales far from 1, also within one call: each row and each value has its own range."""
    torch, binding = gpu
    dt = getattr(torch, dtype)
    x = Batch(torch, dt, 128, 2, 2, 16, [190], [new], seed=7, fused=False)
    for q_by, k_by, v_by, scale in ((1.0, 1.0, 2.0 ** -10, 0.09), (2.0 ** 7, 2.0 ** -8, 2.0 ** 7, 0.1), (2.0 ** -9, 2.0 ** 9, 1.0, 0.05)):
        q = (x.q.float() * q_by).to(dt)
        q[:, 1::2] = (q[:, 1::2].float() * 2.0 ** -4).to(dt)
        y = Batch(torch, dt, 128, 2, 2, 16, [190], [new], seed=7, fused=False)
        y.scales[:, :, 0] = (x.scales[:, :, 0].float() * k_by).to(dt)
        y.scales[:, :, 1] = (x.scales[:, :, 1].float() * v_by).to(dt)
        y.scales[:, :, 1, 3::5] = (y.scales[:, :, 1, 3::5].float() * 2.0 ** -3).to(dt)
        got = binding.apmm_kv_attention(q, *y.args, y.starts_gpu, scale=scale)
        close(torch, got, *y.attention(q, 0, 0, scale))
    if dt == torch.bfloat16:  # beyond what binary16 holds
        y.scales[:, :, 1] = (x.scales[:, :, 1].float() * 2.0 ** 60).to(dt)
        y.scales[:, :, 0] = (x.scales[:, :, 0].float() * 2.0 ** -40).to(dt)
        q = (x.q.float() * 2.0 ** 40).to(dt)
        close(torch, binding.apmm_kv_attention(q, *y.args, y.starts_gpu, scale=0.1), *y.attention(q, 0, 0, 0.1))


@pytest.mark.parametrize("new", [1, 70])
def test_hidden_keys_change_nothing(gpu, new):
    """NaN and the largest numbers in keys and values that no query sees: before the window, behind the end of the last page, in pages of others, in no page."""
    torch, binding = gpu
    x = Batch(torch, torch.float16, 64, 2, 2, 16, [203, 50], [new, 1], seed=5, spare=3, room=2)
    window, sinks = 60, 3
    want = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu, window=window, sinks=sinks)
    seen = torch.zeros(x.scales.shape[0], 16, dtype=torch.bool)
    for b, length in enumerate(x.lengths):
        for j in range(length):
            if j < sinks or j > length - (new, 1)[b] - window:
                seen[int(x.table[b, j // 16]), j % 16] = True
    hidden = ~seen.cuda()
    for bad in (float("nan"), 65504.0, float("inf")):
        scales = torch.where(hidden[:, None, None, :], torch.full_like(x.scales, bad), x.scales)
        got = binding.apmm_kv_attention(x.q, x.codes, scales, *x.args[2:], x.starts_gpu, window=window, sinks=sinks)
        assert torch.equal(got, want), bad
    assert x.table[1, 4:].tolist() == [-1] * (x.table.shape[1] - 4)


@pytest.mark.parametrize("new", [1, 70])
def test_not_a_number_stays_in_its_row(gpu, new):
    """A query that is not finite, and a key that is not (seen by some queries only), reach the results that depend on them and no other."""
    torch, binding = gpu
    x = Batch(torch, torch.bfloat16, 128, 2, 2, 16, [150], [new], seed=6, fused=False)
    want = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu)
    q = x.q.clone()
    q[new // 2, 1, 5], q[0, 3, 7] = float("nan"), float("inf")
    got = binding.apmm_kv_attention(q, *x.args, x.starts_gpu)
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    bad[new // 2, 1] = bad[0, 3] = True
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], want[~bad])
    late = 150 - max(1, new // 2)  # the position of a key that the queries before it do not see
    for which in (0, 1):
        scales = x.scales.clone()
        scales[int(x.table[0, late // 16]), 1, which, late % 16] = float("nan")
        got = binding.apmm_kv_attention(x.q, x.codes, scales, *x.args[2:], x.starts_gpu)
        bad = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
        bad[late - (150 - new):, 2:] = True
        assert bool(torch.isnan(got[bad]).all())
        if which == 0:
            assert torch.equal(got[~bad], want[~bad])
        else:  # (the others' running maximum moves at other keys)
            exact, near = x.attention(x.q, 0, 0, 128 ** -0.5)
            close(torch, got[~bad], exact[~bad.cpu()], near[~bad.cpu()])


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("new, heads, groups", [(16, 2, 1), (5, 1, 3), (90, 2, 2)])
def test_each_row_has_its_own_range(gpu, dtype, new, heads, groups):
    """Very large queries, and keys and values with very large scales that later queries see: the results of the others are as exact as without."""
    torch, binding = gpu
    dt = getattr(torch, dtype)
    D, length = 128, 140
    x = Batch(torch, dt, D, heads, groups, 16, [length], [new], seed=13, fused=False)
    late = length - new // 2
    big = 2.0 ** 11 if dt == torch.float16 else 2.0 ** 100
    exact, near = x.attention(x.q, 0, 0, D ** -0.5)
    before = late - (length - new)  # queries that do not see the key at `late`
    for which in (0, 1):
        scales = x.scales.clone()
        scales[int(x.table[0, late // 16]), :, which, late % 16] = big
        got = binding.apmm_kv_attention(x.q, x.codes, scales, *x.args[2:], x.starts_gpu)
        close(torch, got[:before], exact[:before], near[:before])
    q = x.q.clone()
    q[1::2] *= big / 2 ** 4
    got = binding.apmm_kv_attention(q, *x.args, x.starts_gpu)
    close(torch, got[0::2], exact[0::2], near[0::2])


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("smaller", [4, 9, 14])
def test_queries_of_different_sizes(gpu, dtype, smaller):
    """Rows of a tile whose queries are 2^-smaller of the others': the scores of neither lose bits."""
    torch, binding = gpu
    dt = getattr(torch, dtype)
    x = Batch(torch, dt, 128, 2, 2, 16, [300], [100], seed=17, fused=False)
    q = x.q.clone()
    q[1::3] *= 2.0 ** -smaller
    scale = 128 ** -0.5 * 2.0 ** (smaller // 2)
    got = binding.apmm_kv_attention(q, *x.args, x.starts_gpu, scale=scale)
    close(torch, got, *ref.attention(q, x.codes, x.scales, x.table, x.lengths, x.starts, 0, 0, scale))


@pytest.mark.parametrize("new", [1, 40])
def test_scales_near_the_largest_number(gpu, new):
    """A key scale whose product with the factor of the queries is beyond 32-bit numbers: queries that are zero weigh its key like the others."""
    torch, binding = gpu
    x = Batch(torch, torch.bfloat16, 128, 2, 2, 16, [200], [new], seed=19, fused=False)
    scales = x.scales.clone()
    for at in (3, 45, 77, 140):
        scales[int(x.table[0, at // 16]), :, 0, at % 16] = 2.0 ** 122
    q = x.q.clone()
    q[::2] = 0.0
    got = binding.apmm_kv_attention(q, x.codes, scales, *x.args[2:], x.starts_gpu)
    want, near = ref.attention(q, x.codes, scales, x.table, x.lengths, x.starts, 0, 0, 128 ** -0.5)
    close(torch, got[::2], want[::2], near[::2])


@pytest.mark.parametrize("heads, groups, new", [(64, 1, 700), (100, 1, 1000), (40, 2, 900)])
def test_every_tile_of_a_prompt(gpu, heads, groups, new):
    """Prompts of more tiles of rows than a head has compute units: some rows of each tile and some heads."""
    torch, binding = gpu
    x = Batch(torch, torch.float16, 64, heads, groups, 16, [new + 9], [new], seed=23, fused=False)
    got = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu)
    for h in (0, heads - 1):
        for row in range(0, new, 128 // groups):
            for a in (row, min(row + 128 // groups, new) - 1):
                want, near = ref.attention(x.q[a:a + 1, h * groups:(h + 1) * groups], x.codes[:, h:h + 1], x.scales[:, h:h + 1], x.table, [a + 10], [0, 1], 0, 0, 64 ** -0.5)
                close(torch, got[a:a + 1, h * groups:(h + 1) * groups], want, near)


def test_more_sequences_than_lanes(gpu):
    """Pieces of prompts, single tokens and nothing, in turn, for 150 sequences, some of them long enough to be cut."""
    torch, binding = gpu
    lengths = [(37 * i) % 200 for i in range(150)]
    lengths[7], lengths[100], lengths[149] = 3100, 2500, 2900
    new = [min((1, 40, 0, 1, 1, 3)[i % 6], n) for i, n in enumerate(lengths)]
    x = Batch(torch, torch.float16, 64, 2, 2, 16, lengths, new, seed=29, fused=False)
    got = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu)
    close(torch, got, *x.attention(x.q, 0, 0, 64 ** -0.5))
    got = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu, window=300, sinks=5)
    close(torch, got, *x.attention(x.q, 300, 5, 64 ** -0.5))


def test_pages_that_are_none(gpu):
    """Page numbers outside of the cache: their tokens are not written, read as zeros and are not seen.  Lengths beyond the table, starts that do not fit: nothing outside of the buffers."""
    torch, binding = gpu
    x = Batch(torch, torch.float16, 64, 2, 2, 16, [100, 40], [1, 40], seed=8)
    pages = x.scales.shape[0]
    x.table[0, 1], x.table[0, 3], x.table[1, 0] = -1, pages, 2 ** 31 - 1
    x.args[2] = x.table.cuda()
    codes, scales = x.codes.clone(), x.scales.clone()
    binding.apmm_kv_write(x.k, x.v, *x.args, x.starts_gpu)
    gone = int(x.table[1, 1])
    assert not torch.equal(codes[gone], x.codes[gone])
    k, v = binding.apmm_kv_read(*x.args, x.tokens, x.starts_gpu)
    assert not bool(k[1:17].any()) and not bool(v[1:17].any()) and bool(k[17:].any())
    got = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu)
    close(torch, got, *x.attention(x.q, 0, 0, 64 ** -0.5))
    assert not bool(got[1:17].any())  # they see tokens of the page that is none
    for lengths, starts in (([2 ** 31 - 1, 10 ** 6], [0, 1, 41]), ([-5, -2 ** 31], [0, 1, 41]), ([100, 40], [7, -3, 2 ** 31 - 1]), ([100, 40], [41, 41, 41]), ([100, 2 ** 30], [0, 41, 41])):
        args = x.args[:3] + [torch.tensor(lengths, dtype=torch.int64).to(torch.int32).cuda()]
        s = torch.tensor(starts, dtype=torch.int64).to(torch.int32).cuda()
        binding.apmm_kv_write(x.k, x.v, *args, s)
        binding.apmm_kv_read(*args, x.tokens, s)
        binding.apmm_kv_attention(x.q, *args, s)
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits(gpu):
    """Pages beyond 4 GiB of codes."""
    torch, binding = gpu
    D, heads, ps = 128, 8, 256
    pages = (5 << 30) // (heads * ps * D)
    codes, scales = binding.apmm_kv_cache(pages, ps, heads, D, torch.float16)
    x = Batch(torch, torch.float16, D, heads, 1, ps, [300, 520], [300, 1], seed=9)
    far = [pages - 1 - 7 * i for i in range(x.scales.shape[0])]
    codes[far], scales[far] = x.codes, x.scales
    table = torch.where(x.table >= 0, torch.tensor(far, dtype=torch.int32)[x.table.long()], x.table).cuda()
    want = binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu)
    assert torch.equal(binding.apmm_kv_attention(x.q, codes, scales, table, *x.args[3:], x.starts_gpu), want)
    binding.apmm_kv_write(x.k, x.v, *x.args, x.starts_gpu)
    binding.apmm_kv_write(x.k, x.v, codes, scales, table, *x.args[3:], x.starts_gpu)
    assert torch.equal(codes[far], x.codes) and torch.equal(scales[far], x.scales)
    for a, b in zip(binding.apmm_kv_read(codes, scales, table, *x.args[3:], x.tokens, x.starts_gpu), binding.apmm_kv_read(*x.args, x.tokens, x.starts_gpu)):
        assert torch.equal(a, b)


def test_one_page_for_a_long_sequence(gpu):
    """A page as long as the context, and pages shared by two sequences."""
    torch, binding = gpu
    x = Batch(torch, torch.float16, 128, 2, 2, 1024, [1000, 1], [1, 1], seed=10)
    x.table[1, 0] = x.table[0, 0]
    x.args[2] = x.table.cuda()
    x.lengths[1] = 513
    x.args[3] = torch.tensor(x.lengths, dtype=torch.int32).cuda()
    close(torch, binding.apmm_kv_attention(x.q, *x.args, x.starts_gpu), *x.attention(x.q, 0, 0, 128 ** -0.5))


def test_on_another_stream_and_in_a_graph(gpu):
    """Work goes to the current stream; a step of a serving loop (write, then attention) captured once and replayed with other inputs and lengths."""
    torch, binding = gpu
    lengths = [100, 37, 260]
    x = Batch(torch, torch.float16, 128, 4, 2, 16, [n + 3 for n in lengths], [1, 1, 1], seed=11)
    held = torch.tensor(lengths, dtype=torch.int32).cuda()
    out = torch.zeros_like(x.q.contiguous())
    work = torch.empty(max(1, binding.apmm_kv_attention_workspace_bytes(3, 8, *x.args)), dtype=torch.uint8, device="cuda")
    q, k, v = x.q.contiguous(), x.k.contiguous(), x.v.contiguous()

    def step():
        binding.apmm_kv_write(k, v, x.codes, x.scales, x.args[2], held)
        binding.apmm_kv_attention(q, x.codes, x.scales, x.args[2], held, out=out, workspace=work)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    eager = (x.codes.clone(), x.scales.clone(), out.clone())
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, (x.codes, x.scales, out)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in range(3):
        held += 1
        q.copy_(torch.roll(q, 1, 0))
        k.copy_(torch.roll(k, 1, 2))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), x.codes.clone(), x.scales.clone()
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, x.codes, x.scales)))


def test_nothing_to_do(gpu):
    torch, binding = gpu
    codes, scales = binding.apmm_kv_cache(1, 16, 2, 64)
    none = torch.empty((0,), dtype=torch.int32, device="cuda")
    table = torch.empty((0, 1), dtype=torch.int32, device="cuda")
    q = torch.empty((0, 4, 64), dtype=torch.float16, device="cuda")
    assert binding.apmm_kv_attention(q, codes, scales, table, none).shape == (0, 4, 64)
    binding.apmm_kv_write(q[:, :2], q[:, 2:], codes, scales, table, none)
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    two = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert binding.apmm_kv_attention(q, codes, scales, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), one, two).numel() == 0
    assert binding.apmm_kv_read(codes, scales, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), one, 0, two)[0].shape == (0, 2, 64)


def test_refusals(gpu):
    torch, binding = gpu
    x = Batch(torch, torch.float16, 64, 2, 2, 16, [40], [1], seed=12)
    c, s, t, n = x.args

    def refused(kind, fn, *args, status=None, **kw):
        with pytest.raises(kind) as err:
            fn(*args, **kw)
        if status is not None:
            assert err.value.status == status
    before = c.clone()
    for args in ((x.q.float(), c, s, t, n), (x.q, c.int(), s, t, n), (x.q, c, s.float(), t, n), (x.q, c, s, t.long(), n), (x.q, c, s, t, n.long()), (x.q.cpu(), c, s, t, n),
                 (x.q, c, s, t.cpu(), n), (x.q[0], c, s, t, n), (x.q[:, :, :32], c, s, t, n), (x.q.bfloat16(), c, s, t, n), (x.q, c[:, :1], s, t, n), (x.q, c, s, t, n[:0])):
        refused(ValueError, binding.apmm_kv_attention, *args)
    refused(binding.ApmmError, binding.apmm_kv_attention, x.q[:, :3], c, s, t, n, status=1)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(window=-1), dict(sinks=-1)):
        refused(binding.ApmmError, binding.apmm_kv_attention, x.q, c, s, t, n, status=1, **kw)
    refused(binding.ApmmError, binding.apmm_kv_attention, x.q, c, s, t, n, status=2, window=2 ** 30 + 1)
    wide = torch.full((1, 1 << 20), -1, dtype=torch.int32, device="cuda")  # room for a sequence whose keys may be cut
    assert binding.apmm_kv_attention_workspace_bytes(1, 4, c, s, wide, n) > 16
    refused(binding.ApmmError, binding.apmm_kv_attention, x.q, c, s, wide, n, status=4, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    refused(ValueError, binding.apmm_kv_write, x.k, x.v[:, :1], c, s, t, n)
    refused(ValueError, binding.apmm_kv_write, x.q, x.v, c, s, t, n)
    refused(ValueError, binding.apmm_kv_read, c, s, t, n, 2)
    refused(ValueError, binding.apmm_kv_read, c, s, t, n, 1, k_out=x.q)
    torch.cuda.synchronize()
    assert torch.equal(c, before)
