"""4-bit weights on the GPU against the text in 64 bits (quant_reference): every code and scale, what they read as, and products.

Products are checked in two ways. With whole-numbered inputs and scales that are powers of two every sum is exact in fp32, so the
result is the exact one, rounded once to the output's type. With random inputs the bound is
  |error| <= S * (17 * G / 16 * 2^-23 + (cols / G + 16) * 2^-24) + half a step of the output's type,  S = sum |scale code x|:
a product of 16 columns adds 17 numbers and may lose the last of 24 bits of the largest for each, G / 16 such products make a group's
sum; the groups' sums are added with one rounding each, then those of the warps and the parts of x.
"""
import numpy as np
import pytest
import torch

import quant_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def lc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2009_13003_b200 import binding

    binding.lib()
    return binding


def random_weights(rows, cols, seed, dtype=torch.float32, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randn(rows, cols + pad, generator=g, device=DEV) * torch.exp(2 * torch.randn(rows, 1, generator=g, device=DEV))
    return w.to(dtype)[:, :cols]


def whole_weights(rows, cols, group, seed):
    """Codes -7 ... 7 times a power of two per group, 7 among them."""
    r = np.random.RandomState(seed)
    codes = r.randint(-7, 8, (rows, -(-cols // group) * group))
    codes[:, ::group] = 7
    scale = np.repeat(2.0 ** r.randint(-2, 3, (rows, codes.shape[1] // group)), group, axis=1)
    return (codes * scale)[:, :cols].astype(np.float32)


def check_against_text(q4, w):
    """Every code and scale of the buffer, those that fill it up included."""
    x = w.double().cpu().numpy()
    codes, scales = ref.quantize(x, 4, q4.group)
    got, got_scales = ref.q4_unpack(q4.data.cpu().numpy(), q4.rows, q4.cols, q4.group)
    want = np.zeros_like(got)
    want[: q4.rows, : q4.cols] = codes
    want_scales = np.zeros_like(got_scales)
    want_scales[: q4.rows, : scales.shape[1]] = scales
    assert np.array_equal(got_scales, want_scales)
    assert np.array_equal(got, want)
    return codes, scales


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 31, 0), (16, 128, 0), (17, 200, 0), (33, 257, 1), (40, 1000, 8), (257, 96, 3), (5, 4096, 0)])
def test_codes_scales_and_values(lc, group, kind, rows, cols, pad):
    w = random_weights(rows, cols, rows * cols, TYPES[kind], pad)
    q4 = lc.q4_quantize(w, group)
    codes, scales = check_against_text(q4, w)
    want = torch.from_numpy(ref.values(codes, scales, group))
    for out in TYPES.values():
        got = lc.q4_read(q4, dtype=out).cpu()
        assert torch.equal(got, want.to(torch.float32).to(out)), out  # float32 holds the values, so this rounds once


def test_a_large_matrix(lc):
    w = random_weights(2050, 3001, 5)
    check_against_text(lc.q4_quantize(w, 64), w)


@pytest.mark.parametrize("group", [32, 128])
def test_borders_and_small_and_large_magnitudes(lc, group):
    r = np.random.RandomState(1)
    rows = [np.zeros(512)]
    for s in (1.0, 2.0 ** -126, 2.0 ** -125, 2.0 ** 125, 1.0078125, 1.9921875):  # scales of 8 bits
        half = r.randint(-14, 15, 512) / 2.0 * s  # on borders wherever the code is odd
        half[::group] = 7 * s
        rows.append(half)
        near = np.nextafter(half.astype(np.float32), np.float32(0) if s > 1 else np.float32(3e38))
        near[::group] = np.float32(7 * s)
        rows.append(near)
    for k in (2.0 ** -149, 2.0 ** -140, 2.0 ** -127, 2.0 ** -124):  # the scale falls to 0 between them
        rows.append(r.randint(-9, 10, 512) * k)
    rows.append(r.uniform(-1, 1, 512) * 3.4e38)
    # quotients by 7 next to the middle between two scales
    base = (np.float32(1.0) + (2 * np.arange(512) + 1).astype(np.float32) * np.float32(2.0 ** -9)) * np.float32(7)
    rows += [np.nextafter(base, np.float32(0)), base, np.nextafter(base, np.float32(100))]
    w = torch.from_numpy(np.stack(rows).astype(np.float32)).to(DEV)
    check_against_text(lc.q4_quantize(w, group), w)
    # a group for each of the quotients
    w = torch.from_numpy(np.concatenate(rows[-3:]).astype(np.float32)[:, None]).to(DEV)
    check_against_text(lc.q4_quantize(w, group), w)


def test_inf_and_nan_are_reported_and_stay_in_their_group(lc):
    for bad in (float("inf"), -float("inf"), float("nan")):
        w = random_weights(40, 300, 7)
        w[21, 70] = bad
        q4, ws = lc.alloc_q4(40, 300, 64, DEV), lc.alloc_workspace(0, DEV)
        lc.q4_quantize_async(w, q4, ws)
        assert lc.last_status(ws) == lc.ERR_NONFINITE
        check_against_text(q4, w)
        got = lc.q4_read(q4)
        assert bool(got[21, 64:128].isnan().all()) and int(got.isnan().sum()) == 64
        y = lc.q4_matvec(q4, torch.ones(2, 300, device=DEV))
        assert bool(y[:, 21].isnan().all()) and int(y.isnan().sum()) == 2
        with pytest.raises(lc.LCError) as e:
            lc.q4_quantize(w, 64)
        assert e.value.code == lc.ERR_NONFINITE
        w[21, 70] = 0.0
        lc.q4_quantize_async(w, q4, ws)  # the word is cleared
        assert lc.last_status(ws) == lc.OK


SHAPES = [(1, 1, 1), (16, 128, 1), (17, 33, 2), (120, 400, 1), (31, 129, 5), (64, 1024, 8), (100, 1000, 9), (48, 640, 16), (33, 2049, 17), (1000, 512, 32),
          (20, 300, 33), (16, 256, 64), (40, 500, 65), (24, 384, 150), (2048, 2048, 1), (9, 20000, 3), (50, 9000, 40)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(TYPES))
def test_products_of_whole_numbers_are_exact(lc, group, kind):
    for i, (rows, cols, tokens) in enumerate(SHAPES):
        w = whole_weights(rows, cols, group, i)
        r = np.random.RandomState(100 + i)
        x = r.randint(-4, 5, (tokens, cols + 3))  # |sum| <= 20000 * 4 * 7 * 4 = 2.24e6: exact in fp32, in quarters
        wide = torch.from_numpy(x.astype(np.float32)).to(TYPES[kind]).to(DEV)
        want = torch.from_numpy(x[:, :cols].astype(np.float64) @ w.astype(np.float64).T).to(torch.float32)
        q4 = lc.q4_quantize(torch.from_numpy(w).to(DEV), group)
        for xs in (wide[:, :cols], wide[:, :cols].contiguous()):
            canary = torch.full((tokens + 2, rows + 5), 77.0, device=DEV)
            lc.q4_matvec(q4, xs, canary[1:-1, :rows])
            got = canary.cpu()
            assert torch.equal(got[1:-1, :rows], want), (rows, cols, tokens)
            got[1:-1, :rows] = 77.0
            assert bool((got == 77.0).all())
            same = lc.q4_matvec(q4, xs)
            assert same.dtype == TYPES[kind] and torch.equal(same.cpu(), want.to(TYPES[kind]))


def half_step(y, kind):
    info = torch.finfo(TYPES[kind])
    return torch.maximum(y.abs() * (info.eps / 2), torch.tensor(info.tiny * info.eps / 2, dtype=torch.float64))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,tokens", [(300, 5003, 1), (130, 4096, 4), (67, 1111, 20), (257, 3000, 64)])
def test_products_of_random_numbers(lc, group, kind, rows, cols, tokens):
    w = random_weights(rows, cols, 3)
    q4 = lc.q4_quantize(w, group)
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(tokens, cols, generator=g, device=DEV).to(TYPES[kind])
    codes, scales = ref.quantize(w.double().cpu().numpy(), 4, group)
    v = torch.from_numpy(ref.values(codes, scales, group))
    xd = x.double().cpu()
    want, size = xd @ v.T, xd.abs() @ v.abs().T
    bound = size * (17 * group / 16 * 2.0 ** -23 + (cols / group + 16) * 2.0 ** -24)
    for out in (None, torch.empty(tokens, rows, device=DEV)):
        got = lc.q4_matvec(q4, x, out)
        step = half_step(want, kind if out is None else "fp32")
        assert bool(((got.double().cpu() - want).abs() <= bound + step * (1 + 1e-3)).all())
    assert torch.equal(lc.q4_matvec(q4, x), lc.q4_matvec(q4, x))


def test_all_bits_of_an_fp32_vector_count(lc):
    # one weight of 1 per row: the product is the vector's value itself, at every magnitude
    n = 256
    w = torch.zeros(n, n, device=DEV)
    w.fill_diagonal_(7.0)
    r = np.random.RandomState(5)
    x = (r.randint(1 << 23, 1 << 24, n) * 2.0 ** r.randint(-120, 80, n) * r.choice([-1, 1], n)).astype(np.float32)
    q4 = lc.q4_quantize(w, 32)  # scale 1, code 7
    got = lc.q4_matvec(q4, torch.from_numpy(x).to(DEV)).cpu().numpy()
    # 7 * x needs 27 bits: the parts' products are exact, their sum is rounded twice at most
    assert np.all(np.abs(got.astype(np.float64) - 7.0 * x.astype(np.float64)) <= 2.0 ** -23 * np.abs(7.0 * x.astype(np.float64)))
    got = lc.q4_matvec(lc.q4_quantize(w / 7.0 * 4.0, 32), torch.from_numpy(x).to(DEV)).cpu().numpy()
    s = ref.bf16_values(ref.bf16_bits(np.float64(4.0) / 7.0))
    want = 7.0 * s * x.astype(np.float64)
    assert np.all(np.abs(got.astype(np.float64) - want) <= 2.0 ** -22 * np.abs(want))


@pytest.mark.parametrize("tokens", [1, 3, 20])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_small_and_large_weights_and_vectors(lc, kind, tokens):
    rows, cols, group = 70, 900, 64
    bound = 17 * group / 16 * 2.0 ** -23 + (cols / group + 16) * 2.0 ** -24
    for w_exp, x_exp in ((-100, 0), (-100, 60), (90, 0), (90, -60), (0, 46), (0, 50), (0, 100), (-60, 100), (0, -70), (100, -70)):
        w = random_weights(rows, cols, 21) * 2.0 ** w_exp
        x = (torch.randn(tokens, cols, device=DEV) * 2.0 ** x_exp).to(TYPES[kind])
        x[0, 5] *= 16.0
        got = lc.q4_matvec(lc.q4_quantize(w, group), x, torch.empty(tokens, rows, device=DEV)).double().cpu()
        codes, scales = ref.quantize(w.double().cpu().numpy(), 4, group)
        v, xd = torch.from_numpy(ref.values(codes, scales, group)), x.double().cpu()
        # a sum of codes and x may lose what lies below 2^-96, a group's scale times that
        lost = 2.0 ** -95 * 16 * torch.from_numpy(ref.bf16_values(scales)).sum(-1)
        assert bool(((got - xd @ v.T).abs() <= (xd.abs() @ v.abs().T) * bound + lost + 2.0 ** -149).all()), (w_exp, x_exp)


@pytest.mark.parametrize("kind", list(TYPES))
def test_inf_and_nan_in_a_vector(lc, kind):
    w = torch.ones(40, 200, device=DEV)
    w[::2] = -1.0
    q4 = lc.q4_quantize(w, 64)
    x = torch.ones(5, 210, device=DEV, dtype=TYPES[kind])
    x[:, 200:] = float("nan")  # behind the vectors: not read into the sums
    x[1, 3], x[2, 150], x[3, 199] = float("inf"), float("nan"), -float("inf")
    y = lc.q4_matvec(q4, x[:, :200]).float().cpu()
    sign = torch.where(torch.arange(40) % 2 == 0, -1.0, 1.0)
    assert bool((y[0].abs() < 300).all()) and torch.equal(y[0], y[4])
    assert torch.equal(y[1], sign * float("inf")) and bool(y[2].isnan().all()) and torch.equal(y[3], -sign * float("inf"))
    if kind == "fp32":  # a NaN whose upper half alone would be an Inf
        x[2, 150] = torch.tensor(0x7F800001, dtype=torch.int32).view(torch.float32)
        assert bool(lc.q4_matvec(q4, x[:, :200])[2].isnan().all())


def test_one_vector_for_all_tokens_and_nothing_to_do(lc):
    w = random_weights(50, 300, 9)
    q4 = lc.q4_quantize(w, 32)
    x = torch.randn(300, device=DEV)
    one = lc.q4_matvec(q4, x)
    assert one.shape == (50,) and torch.equal(lc.q4_matvec(q4, x.expand(6, 300)), one.expand(6, 50))
    assert lc.q4_matvec(q4, x.new_empty(0, 300)).shape == (0, 50)
    empty = lc.q4_quantize(torch.empty(0, 300, device=DEV), 32)
    assert empty.data.numel() == 0 and lc.q4_matvec(empty, x).shape == (0,) and lc.q4_read(empty).shape == (0, 300)
    none = lc.q4_quantize(torch.empty(50, 0, device=DEV), 32)
    assert torch.equal(lc.q4_matvec(none, torch.empty(3, 0, device=DEV)), torch.zeros(3, 50, device=DEV)) and lc.q4_read(none).shape == (50, 0)


@pytest.mark.parametrize("kind,tokens", [("fp32", 655351), ("fp32", 1048576), ("bf16", 1048576)])
def test_as_many_vectors_as_allowed(lc, kind, tokens):
    """Up to LC_Q4_MAX_TOKENS vectors, more passes than a grid has rows; whole numbers, so that every sum is exact."""
    w = whole_weights(2, 32, 32, 5)
    x = (torch.arange(tokens * 32, device=DEV).view(tokens, 32) % 9 - 4).to(TYPES[kind])
    got = lc.q4_matvec(lc.q4_quantize(torch.from_numpy(w).to(DEV), 32), x, torch.empty(tokens, 2, device=DEV))
    want = (x.double() @ torch.from_numpy(w.astype(np.float64)).to(DEV).T).float()
    assert torch.equal(got, want)


def test_on_another_stream_and_in_a_graph(lc):
    w, x = random_weights(200, 700, 11), torch.randn(3, 700, device=DEV)
    q4, ws = lc.alloc_q4(200, 700, 64, DEV), lc.alloc_workspace(0, DEV)
    want = lc.q4_matvec(lc.q4_quantize(w, 64), x)
    back, y = torch.empty(200, 700, device=DEV), torch.empty(3, 200, device=DEV)

    def steps():
        lc.q4_quantize_async(w, q4, ws)
        lc.q4_read(q4, back)
        lc.q4_matvec(q4, x, y)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        steps()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    w.mul_(-2.0)  # what the graph reads when it is replayed
    x.mul_(3.0)
    graph.replay()
    assert torch.equal(y, lc.q4_matvec(lc.q4_quantize(w, 64), x)) and torch.equal(back, lc.q4_read(q4)) and lc.last_status(ws) == lc.OK


def test_a_chain_recovered_into_weights(lc, oracle):
    rows, cols = 250, 333
    n = rows * cols
    g = torch.Generator(device=DEV).manual_seed(1)
    base = torch.randn(n, generator=g, device=DEV) * 0.02
    tracked, cur, streams = base.clone(), base.clone(), []
    for _ in range(3):
        cur = cur + torch.randn(n, generator=g, device=DEV) * 1e-3
        s, tracked = lc.compress_update(tracked, cur, 4)
        streams.append(s.clone())
    state = oracle.recover(base.cpu().numpy(), [s.cpu().numpy() for s in streams])
    scratch = torch.empty_like(base)
    q4 = lc.recover_q4(base, streams, rows, 32, scratch=scratch)
    assert np.array_equal(scratch.cpu().numpy().view(np.uint32), state.view(np.uint32))
    check_against_text(q4, torch.from_numpy(state).view(rows, cols))
    # a stream of another size: the status word of the recovery stays
    other = lc.compress(base[: n - 4], cur[: n - 4], 4)
    with pytest.raises(lc.LCError) as e:
        lc.recover_q4(base, [streams[0], other], rows, 32)
    assert e.value.code == lc.ERR_MISMATCH


def test_the_binding_refuses(lc):
    w, x = random_weights(20, 64, 1), torch.randn(2, 64, device=DEV)
    q4, ws = lc.q4_quantize(w, 32), lc.alloc_workspace(0, DEV)
    for call in (lambda: lc.q4_quantize(w.double()), lambda: lc.q4_quantize(w.cpu()), lambda: lc.q4_quantize(w.t()), lambda: lc.q4_quantize(w[0]),
                 lambda: lc.q4_quantize_async(w[:, :63], q4, ws), lambda: lc.q4_matvec(q4, x[:, :60]), lambda: lc.q4_matvec(q4, x.cpu()),
                 lambda: lc.q4_matvec(q4, x.requires_grad_()), lambda: lc.q4_matvec(q4, x.detach(), torch.empty(2, 21, device=DEV)),
                 lambda: lc.q4_matvec(q4, x.detach().int()), lambda: lc.q4_read(q4, torch.empty(64, 20, device=DEV))):
        with pytest.raises(ValueError):
            call()
    x = x.detach()
    for call in (lambda: lc.q4_quantize(w, 48), lambda: lc.q4_matvec(q4._replace(group=16), x), lambda: lc.q4_matvec(q4, x, torch.empty(2, 20, device=DEV).half()),
                 lambda: lc.q4_matvec(q4._replace(rows=2000), x)):
        with pytest.raises(lc.LCError):
            call()
