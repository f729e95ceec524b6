"""The K/V store operators on a B200 at values where a rounding, a mask or a factor can show: infinite values, hidden keys,
small probabilities in long ranges, softmax scales at the ends of fp32."""
import math

import numpy as np
import pytest
import torch

import store_reference as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
FORMATS = [("f32", "f32"), ("bf16", "bf16"), ("kv8", "bf16"), ("kv8", "f32")]


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


def _normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _i64(x):
    return torch.tensor(x, dtype=torch.int64, device="cuda")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _store(pkg, fmt, k, v):
    if fmt == "kv8":
        (ck, sk), (cv, sv) = ref.quantise(k), ref.quantise(v)
        store = pkg.H2OStore(*[torch.from_numpy(x).cuda() for x in (ck, cv, sk, sv)])
        return store, ref.values(ck, sk).transpose(1, 0, 2), ref.values(cv, sv).transpose(1, 0, 2)
    return pkg.H2OStore(k.cuda(), v.cuda()), k.double().numpy(), v.double().numpy()


def _attend(store, q, begin, length, n, scale=0.0):
    """Sequences of n tokens each; out and lse."""
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    kw = {} if n == 1 else {"cu_q": _i32([n * i for i in range(len(begin) + 1)]), "max_q": n}
    store.cross_attend(q, _i64(begin), _i32(length), out, max_len=max(length), lse=lse, softmax_scale=scale, **kw)
    assert store.status() == 0
    return out, lse


@pytest.mark.parametrize("fmt", ["f32", "bf16"])  # (8-bit rows have no infinities)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,length", [(1, 50), (1, 3000), (4, 50), (16, 50), (16, 900), (17, 50), (150, 50), (150, 700)])
def test_infinite_values_stay_infinite(pkg, fmt, dim, n, length):
    """A value of +-infinity with a positive probability gives that infinity, whatever the number of query rows; both signs
    in one channel, or a NaN, give NaN.  The sequences: a single key (probability 1), keys of equal logits (probabilities that
    are powers of two), random ones."""
    rows = 4 + 64 + length
    k, v = (_normal(s, rows, 1, dim).to(DT[fmt]) for s in (1, 2))
    k[:68] = 0
    k[68:] *= 0.3
    v[1, 0, 3], v[1, 0, 4] = math.inf, -math.inf
    v[20, 0, 5], v[30, 0, 6], v[31, 0, 6] = math.inf, math.inf, -math.inf
    v[68 + length // 3, 0, ::7], v[68 + length // 2, 0, 1::7] = math.inf, -math.inf
    v[rows - 1, 0, 1], v[rows - 1, 0, 2] = math.inf, math.nan
    store, k64, v64 = _store(pkg, fmt, k, v)
    begin, ln = [1, 4, 68], [1, 64, length]
    q = _normal(3, 3 * n, 1, dim).to(DT[fmt]).cuda()
    out, lse = _attend(store, q, begin, ln, n)
    for b in range(3):
        sl = slice(b * n, b * n + n)
        with np.errstate(invalid="ignore"):
            want = ref.attend(q[sl].double().cpu().numpy(), k64[begin[b]:begin[b] + ln[b]], v64[begin[b]:begin[b] + ln[b]],
                              [ln[b]] * n, float(np.float32(1 / math.sqrt(dim))), fmt, fmt)
            ref.compare(out[sl], want[0], want[2], "out of sequence %d" % b)
        ref.compare(lse[sl], want[1], want[3], "lse of sequence %d" % b)


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("group,n", [(1, 4), (8, 2), (1, 12), (2, 6)])
def test_infinite_own_values_behind_a_prefix(pkg, fmt, group, n):
    """The same among the own rows of sequences that share a prefix: infinite in the last row, so for the last token."""
    dim, pre, own, batch = 64, 40, 30, 3
    rows = pre + own * batch
    k, v = (_normal(s, rows, 1, dim).to(DT[fmt]) for s in (1, 2))
    for b in range(batch):
        v[pre + own * (b + 1) - 1, 0, 5 + b] = math.inf
    store, k64, v64 = _store(pkg, fmt, k, v)
    q = _normal(3, batch * n, group, dim).to(DT[fmt]).cuda()
    for most in (pre, 5000):  # (the bound of a prefix decides how the call is cut)
        out = torch.empty_like(q)
        store.prefix_attend(q, _i64([0]), _i32([pre]), _i64([pre + own * b for b in range(batch)]), _i32([own] * batch), out,
                            max_prefix=most, max_own=own, cu_q=_i32([n * b for b in range(batch + 1)]), max_q=n)
        assert store.status() == 0
        for b in range(batch):
            at = pre + own * b
            kk, vv = (np.concatenate([x[:pre], x[at:at + own]]) for x in (k64, v64))
            last = b * n + n - 1
            want = ref.attend(q[last:last + 1].double().cpu().numpy(), kk, vv, [pre + own], float(np.float32(1 / math.sqrt(dim))), fmt, fmt)
            assert np.isposinf(want[0][0, :, 5 + b]).all()
            ref.compare(out[last:last + 1], want[0], want[2], "last token of sequence %d" % b)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group,n,own", [(1, 5, 30), (1, 16, 40), (1, 40, 100), (2, 90, 200), (1, 150, 700), (1, 300, 300)])
def test_hidden_keys_weigh_nothing(pkg, fmt, q_dtype, dim, group, n, own):
    """Values of the largest magnitudes in the rows of later tokens: tokens before them see nothing of it."""
    pre, rows = 20, 20 + own
    big = 57344.0 if fmt == "kv8" else 3.0e38
    k, v = (_normal(s, rows, 1, dim).to(DT.get(fmt, torch.bfloat16)) for s in (1, 2))
    v[rows - n + 1:] = big  # the rows of all tokens but the first
    store, k64, v64 = _store(pkg, fmt, k, v)
    q = _normal(3, n, group, dim).to(DT[q_dtype]).cuda()
    for most in (pre, 5000):
        out, lse = torch.empty_like(q), torch.empty((n, group), dtype=torch.float32, device="cuda")
        store.prefix_attend(q, _i64([0]), _i32([pre]), _i64([pre]), _i32([own]), out, max_prefix=most, max_own=own, cu_q=_i32([0, n]),
                            max_q=n, lse=lse)
        assert store.status() == 0
        want = ref.attend(q[:1].double().cpu().numpy(), k64, v64, [rows - n + 1], float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
        ref.compare(out[:1], want[0], want[2], "first token")
        ref.compare(lse[:1], want[1], want[3], "lse of the first token")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,length", [(1, 60), (16, 60), (17, 60), (150, 60), (150, 700)])
def test_keys_with_logits_of_minus_infinity_weigh_nothing(pkg, dim, n, length):
    k, v = (_normal(s, length, 1, dim).bfloat16() for s in (1, 2))
    off = torch.arange(length) % 3 != 0
    k[off, 0, 0] = -math.inf
    v[off] = 3.0e38
    store, k64, v64 = _store(pkg, "bf16", k, v)
    q = _normal(3, n, 1, dim).abs().bfloat16().cuda()
    out, lse = _attend(store, q, [0], [length], n)
    on = ~off.numpy()
    want = ref.attend(q.double().cpu().numpy(), k64[on], v64[on], [int(on.sum())] * n, float(np.float32(1 / math.sqrt(dim))), "bf16", "bf16")
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("q_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [0, 130000])
@pytest.mark.parametrize("tokens,n", [(700, 1), (20000, 20000)])
def test_many_small_probabilities_add_up_on_8_bit_rows(pkg, q_dtype, at, tokens, n):
    """One key with a logit of 26 (base 2) above 2^18 others: each of those weighs 2^-26, all of them 2^-8.  So many query
    rows that the keys are not split.

    Tolerance: the probabilities are f16 operands, off by 2^-11 relative or 2^-25 of their unit where they are subnormal;
    the unit is at most 2^-7 of the largest weight that it has met.  So 2^-32 per key, 2^-11 and the output's 2^-8 of the
    result, and 2^-16 for sums and exponentials."""
    if n > 1 and q_dtype == "f32":
        tokens = n = 300  # (the kernel for float32 queries has no such operand and is slow)
    length, dim = 1 << 18, 64
    code = torch.zeros((1, length, dim), dtype=torch.uint8, device="cuda")
    scale = torch.full((1, length), 127, dtype=torch.uint8, device="cuda")
    vcode = torch.full_like(code, 0x38)  # 1.0
    code[0, at, 0], vcode[0, at] = 0x38, 0
    store = pkg.H2OStore(code, vcode, scale, scale.clone())
    q = torch.zeros((tokens, 1, dim), dtype=DT[q_dtype], device="cuda")
    q[:, 0, 0] = 26.0
    c = math.log(2.0)
    if n == 1:
        out, lse = _attend(store, q, [0] * tokens, [length] * tokens, 1, c)
    else:
        out, lse = _attend(store, q, [0], [length], n, c)
    x = 26.0 * float(np.float32(c))
    others = (length - 1) * math.exp(-x)
    want = others / (1.0 + others)
    got = out.double()
    tol = length * 2.0 ** -32 + want * (2.0 ** -11 + 2.0 ** -8 + 2.0 ** -16)
    assert (got - want).abs().max().item() <= tol, ((got - want).abs().max().item(), tol, want)
    assert (lse.double() - (x + math.log1p(others))).abs().max().item() <= 2.0 ** -16 * x


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("scale", [1e-16, 1e-30, 1e-38, 2e-45])
@pytest.mark.parametrize("n", [1, 20, 70, 150])
def test_tiny_softmax_scales(pkg, fmt, q_dtype, scale, n):
    """Logits of 0 up to rounding: every key weighs the same, and what lies behind the range nothing.  Queries of zeros, tiny
    ones and ordinary ones."""
    dim, length = 64, 37
    k, v = (_normal(s, length + 60, 1, dim).to(DT.get(fmt, torch.bfloat16)) for s in (1, 2))
    store, k64, v64 = _store(pkg, fmt, k, v)
    q = _normal(3, 3 * n, 1, dim)
    q[:n] = 0.0
    q[n:2 * n] *= 2.0 ** -110
    q = q.to(DT[q_dtype]).cuda()
    out, lse = _attend(store, q, [0] * 3, [length] * 3, n, scale)
    want = ref.attend(q.double().cpu().numpy(), k64[:length], v64[:length], [length] * (3 * n), float(np.float32(scale)), fmt, q_dtype)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("q_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 20, 70, 150])
def test_scale_bytes_outside_the_format_count_as_the_nearest_inside(pkg, q_dtype, dim, n):
    """A caller's own codes and scales: every byte as a scale, read back and attended."""
    rows = 256
    g = torch.Generator().manual_seed(5)
    code = torch.randint(0, 0x7F, (2, 1, rows, dim), generator=g, dtype=torch.uint8) | (torch.randint(0, 2, (2, 1, rows, dim), generator=g, dtype=torch.uint8) << 7)
    byte = torch.stack([torch.randperm(256, generator=g), torch.randperm(256, generator=g)]).to(torch.uint8).view(2, 1, rows)
    store = pkg.H2OStore(code[0].cuda(), code[1].cuda(), byte[0].cuda(), byte[1].cuda())
    k64, v64 = (ref.values(code[i], byte[i].clamp(112, 134)).transpose(1, 0, 2) for i in range(2))
    back = [torch.empty((rows, 1, dim), dtype=DT[q_dtype], device="cuda") for _ in range(2)]
    store.read(*back)
    for got, want in zip(back, (k64, v64)):
        np.testing.assert_array_equal(got.double().cpu().numpy(), want)
    q = (_normal(4, n, 1, dim) * 1e-4).to(DT[q_dtype]).cuda()
    out, lse = _attend(store, q, [0], [rows], n)
    want = ref.attend(q.double().cpu().numpy(), k64, v64, [rows] * n, float(np.float32(1 / math.sqrt(dim))), "kv8", q_dtype)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 16, 17, 150, 300])
@pytest.mark.parametrize("steps", [6, 12, 39])
def test_large_values_and_growing_logits_do_not_overflow(pkg, dim, n, steps):
    """Values of 2^99, and single keys whose logits are `steps` (base 2), twice that, ... above the others': sums are kept
    relative to a maximum that may lag, but not by so much that fp32 ends."""
    length = 500
    k, v = torch.zeros((length, 1, dim)), torch.full((length, 1, dim), 2.0 ** 99)
    k[150::100, 0, 0] = steps * torch.arange(1.0, 5.0)
    v[::2] *= -0.5
    store, k64, v64 = _store(pkg, "bf16", k.bfloat16(), v.bfloat16())
    q = torch.zeros((n, 1, dim), dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 1.0
    c = math.log(2.0)
    out, lse = _attend(store, q, [0], [length], n, c)
    want = ref.attend(q.double().cpu().numpy(), k64, v64, [length] * n, float(np.float32(c)), "bf16", "bf16")
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")
