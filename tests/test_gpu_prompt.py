"""tv_prompt_attention against the plain 64-bit form: packed sequences of all kinds of lengths,
earlier keys, more queries than keys, grouped heads, odd head sizes, strides, garbage in places
that a query does not see (needs an MI355X)."""

import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2505_12398_amd as tv
from oracle import decoding as D

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    tv.load_library()
    yield


def starts(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)


def inputs(nq, nk, heads, kv_heads, dim, dtype="bf16", seed=0, before=0, behind=0, packed=None,
           scale_q=1.0):
    """Device arguments of sequences of nq queries and nk keys (None: the same), ``before`` and
    ``behind`` them rows of no sequence, which hold garbage."""
    g = torch.Generator().manual_seed(seed)
    same = nk is None
    tq = before + sum(nq) + behind
    tk = tq if same else before + sum(nk) + behind

    def normal(rows, h):
        x = torch.randn((rows, h, dim), generator=g)
        x[:before], x[rows - behind:] = float("nan"), float("inf")
        return x
    q, k, v = normal(tq, heads) * scale_q, normal(tk, kv_heads), normal(tk, kv_heads)
    if same:
        qkv = torch.cat([q, k, v], dim=1).to(TYPES[dtype]).to(DEV)
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    else:
        q = q.to(TYPES[dtype]).to(DEV)
        kv = torch.cat([k, v], dim=1).to(TYPES[dtype]).to(DEV)
        k, v = kv[:, :kv_heads], kv[:, kv_heads:]
    call = dict(q=q, k=k, v=v, q_start=torch.as_tensor(starts(nq, before), device=DEV),
                scale=float(np.float32(dim ** -0.5)))
    if not same:
        call["k_start"] = torch.as_tensor(starts(nk, before), device=DEV)
    return call


def exact(call):
    """out, sum p |v - out|, sum p |v|, the largest scale sum |q k| and |v| that a query sees, and how
    many keys: per sequence, in 64 bits on the device."""
    q, k, v = (call[x].double() for x in "qkv")
    qs = call["q_start"].tolist()
    ks = call["k_start"].tolist() if "k_start" in call else qs
    G = q.shape[1] // k.shape[1]
    out = torch.full_like(q, float("nan"))
    far, mass = torch.zeros_like(q), torch.zeros_like(q)
    big, most = (torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV) for _ in range(2))
    count = torch.zeros(q.shape[0], dtype=torch.float64, device=DEV)
    for b in range(len(qs) - 1):
        nq, nk = qs[b + 1] - qs[b], ks[b + 1] - ks[b]
        rows = slice(qs[b], qs[b + 1])
        see = torch.ones((nq, nk), dtype=torch.bool, device=DEV).tril(nk - nq)
        count[rows] = see.sum(1)
        for h in range(q.shape[1]):
            if nq == 0:
                continue
            if nk == 0:
                out[rows, h] = 0
                continue
            kh, vh = (x[ks[b]:ks[b + 1], h // G].contiguous() for x in (k, v))
            qh = q[rows, h].contiguous()
            s = (qh @ kh.T.contiguous() * call["scale"]).masked_fill(~see, -float("inf"))
            p = torch.exp(s - s.amax(1, keepdim=True).clamp(min=-1e300))
            p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
            o = p @ vh
            out[rows, h] = o
            mass[rows, h] = p @ vh.abs()
            # sum p |v - out| <= sqrt(sum p (v - out)^2)
            far[rows, h] = ((p @ vh.square()) - o.square() * (count[rows, None] > 0)).clamp(min=0).sqrt()
            big[rows, h] = (qh.abs() @ kh.abs().T.contiguous() * call["scale"]).masked_fill(~see, 0).amax(1)
            most[rows, h] = vh.abs().amax()
    return out, far, mass, big, most, count


def tolerance(e, dtype, dim):
    """The output's rounding; that of every weight to the same type, the sum of the rounded ones
    dividing: half a step of sum p |v - out| (1.1: of the second order); fp32: the score's dot
    product ((dim + 8) roundings of sum |q k|, 4 times, for e^(x + d) = e^x (1 + d) in numerator and
    sum), the exponent and the frame (16 roundings), sums over the keys; fp16 weights below 2^-21 of
    the largest are rounded to multiples of 2^-31 of it: half of that a key, of |v - out| <= 2 max |v|,
    and outputs below fp16's normal range to multiples of 2^-24."""
    out, far, mass, big, most, count = e
    half, fp = torch.finfo(TYPES[dtype]).eps / 2, 2.0 ** -24
    n = count[:, None, None]
    tol = half * out.abs() + 1.1 * half * far + \
        (4 * (dim + 8) * fp * big[..., None] + 16 * fp + 2 * n * fp) * mass
    if dtype == "f16":
        tol = tol + 2.0 ** -31 * n * most[..., None] + 2.0 ** -25
    return tol + 1e-30


def check(call, dtype="bf16", out=None):
    got = tv.prompt_attention(**call) if out is None else out
    e = exact(call)
    rows = slice(int(call["q_start"][0]), int(call["q_start"][-1]))
    err = (got.double() - e[0])[rows].abs()
    tol = tolerance(e, dtype, got.shape[2])[rows]
    bad = ~(err <= tol)
    assert not bad.any(), (float((err / tol).nan_to_num(1e9).max()), bad.nonzero()[:4].tolist())
    return got


def test_reference_is_the_oracle():
    call = inputs([5, 0, 7, 3], [9, 2, 3, 3], 4, 2, 16)
    e = exact(call)
    q, k, v = (call[x].double().cpu().numpy() for x in "qkv")
    for b, (a, z, x, y) in enumerate(((0, 5, 0, 9), (5, 5, 9, 11), (5, 12, 11, 14), (12, 15, 14, 17))):
        out, mass, big = D.prompt_attention(q[a:z], k[x:y], v[x:y], call["scale"])
        for want, got in ((out, e[0]), (mass, e[2]), (big, e[3])):
            np.testing.assert_allclose(got[a:z].cpu().numpy(), want, atol=1e-12)


LENGTHS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 100, 0, 129, 257]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 2), (8, 1), (6, 2), (5, 1), (32, 1)])
def test_lengths_and_heads(dtype, heads, kv_heads):
    check(inputs(LENGTHS, None, heads, kv_heads, 128, dtype), dtype)


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 64, 72, 80, 88, 96, 104, 112, 120, 128])
def test_head_sizes(dim):
    dtype = "f16" if dim % 16 else "bf16"
    check(inputs([70, 3, 150], None, 6, 2, dim, dtype), dtype)


@pytest.mark.parametrize("n", [1, 2, 7, 15, 16, 17, 32, 48, 90, 300])
def test_one_sequence(n):
    check(inputs([n], None, 4, 2, 64))
    check(inputs([n], None, 4, 1, 128, "f16"), "f16")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (8, 2, 128), (3, 1, 80)])
def test_earlier_keys(dtype, heads, kv_heads, dim):
    """Pieces of prompts behind what came before, single tokens among them; sequences with more
    queries than keys, whose first rows see nothing, and without any keys."""
    nq = [1, 40, 64, 5, 100, 33, 7, 0, 1]
    nk = [500, 41, 64, 300, 60, 1, 0, 20, 1]
    call = inputs(nq, nk, heads, kv_heads, dim, dtype)
    got = check(call, dtype)
    at = starts(nq)
    for b in range(len(nq)):
        none = max(0, nq[b] - nk[b])
        assert not got[at[b]:at[b] + none].any()


@pytest.mark.parametrize("heads,kv_heads,n", [(32, 8, 1100), (32, 8, 2100), (8, 8, 4200),
                                              (64, 8, 1030), (16, 2, 4100)])
def test_wide_blocks(heads, kv_heads, n):
    """Enough rows that workgroups take 128 and 256 of them."""
    check(inputs([n, 37, n // 2], None, heads, kv_heads, 64, seed=n))
    check(inputs([n], None, heads, kv_heads, 128, "f16", seed=n), "f16")


def test_wide_blocks_behind_earlier_keys():
    check(inputs([900, 1500, 64], [3001, 1500, 5000], 32, 8, 128))
    check(inputs([2500], [6000], 40, 8, 80, "f16"), "f16")


def test_many_sequences():
    """More sequences than the plan holds at a time, most of them short, empty ones among them."""
    rng = np.random.default_rng(3)
    nq = rng.integers(0, 9, 2500)
    nq[[0, 1023, 1024, 2047, 2499]] = 40, 0, 70, 33, 1
    check(inputs(nq.tolist(), None, 4, 2, 32))
    nk = nq + rng.integers(-3, 30, 2500).clip(min=-nq)
    check(inputs(nq.tolist(), nk.tolist(), 4, 2, 32, "f16"), "f16")


def test_more_items_than_the_plan_has_threads():
    check(inputs([37, 3500, 700], None, 64, 1, 64))


def test_rows_of_no_sequence():
    """Garbage before the first and behind the last sequence reaches none, and its outputs stay."""
    call = inputs([20, 75], None, 4, 2, 64, before=3, behind=40)
    out = torch.full((138, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    check(call, out=tv.prompt_attention(**call, out=out))
    assert (out[:3] == 7.0).all() and (out[98:] == 7.0).all()
    call = inputs([20, 75, 1], [50, 75, 9], 4, 2, 64, before=2, behind=33)
    out = torch.full((131, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    check(call, out=tv.prompt_attention(**call, out=out))
    assert (out[:2] == 7.0).all() and (out[98:] == 7.0).all()


@pytest.mark.parametrize("group,n", [(1, 200), (4, 200), (4, 2200)])
def test_garbage_behind_a_query(group, n):
    """NaN in later keys and values, infinities too, change no bit of the queries before them."""
    call = inputs([n, 50], None, 8 * group, 8, 64)
    clean = check(call)
    for at in (n - 1, n - 37, n // 2, 1):
        k, v = call["k"].clone(), call["v"].clone()
        k[at:n] = float("nan")
        v[at:n] = float("inf")
        v[at:n:2] = float("nan")
        got = tv.prompt_attention(call["q"], k, v, call["q_start"], call["scale"])
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[n:], clean[n:])
        assert torch.isnan(got[at:n]).all()


@pytest.mark.parametrize("nk", [150, 400])
def test_infinite_values(nk):
    """An infinite value is infinite in its own dimension, for the queries that see it."""
    call = inputs([150, 20], [nk, 20], 8, 2, 64)
    clean = check(call)
    for at in (0, 31, nk - 150, nk - 149, nk - 100, nk - 1):
        v = call["v"].clone()
        v[at, :, 3] = float("inf")
        got = tv.prompt_attention(**dict(call, v=v, k=call["k"].clone()))
        sees = torch.arange(150, device=DEV) + nk - 150 >= at
        assert (got[:150][sees][..., 3] == float("inf")).all()
        assert torch.equal(got[:150][~sees], clean[:150][~sees]) and torch.equal(got[150:], clean[150:])
        rest = [d for d in range(64) if d != 3]
        assert torch.equal(got[..., rest], clean[..., rest])


@pytest.mark.parametrize("dtype,dim,heads,n,earlier", [
    ("bf16", 64, 4, 40, 160), ("f16", 64, 4, 200, 0), ("f16", 64, 32, 30, 3001), ("f16", 64, 32, 512, 1490),
    ("f16", 64, 32, 2500, 0), ("bf16", 128, 8, 100, 400), ("f16", 128, 8, 300, 700), ("f16", 80, 32, 1100, 0)])
def test_infinite_values_of_hardly_any_weight(dtype, dim, heads, n, earlier):
    """A value's weight is above 0 however low its score: infinity and NaN reach their own element of the
    queries that see them, and no other bit, where the weight rounds to 0 as well, and where later keys
    score much higher."""
    call = inputs([n, 9], [n + earlier, 9], heads, 2, dim, dtype, seed=n)
    q, k = call["q"].clone(), call["k"].clone()
    q[..., 0] = 1.0 / call["scale"]
    low = [0, 5, earlier // 2, earlier + n // 3, earlier + n - 1]
    nk = n + earlier
    k[:nk, :, 0] = torch.linspace(0.0, 70.0, nk, device=DEV)[:, None].to(k.dtype)   # 70 apart and
    k[low, :, 0] = -200.0                                                           # 200
    call = dict(call, q=q, k=k)
    clean = tv.prompt_attention(**dict(call, v=call["v"].clone()))
    assert bool(clean.isfinite().all())
    bad = ((0, 3, "inf"), (5, 4, "-inf"), (earlier // 2, 3, "inf"), (earlier + n // 3, 6, "nan"),
           (earlier + n - 1, 7, "inf"), (nk // 3, 0, "-inf"), (1, dim - 1, "nan"))
    for some in [(x,) for x in bad] + [bad]:
        v = call["v"].clone()
        want = clean.clone()
        for at, d, x in some:
            v[at, :, d] = float(x)
            sees = torch.arange(n, device=DEV) + earlier >= at
            want[:n, :, d][sees] += float(x)
        got = tv.prompt_attention(**dict(call, v=v))
        assert torch.equal(got.isnan(), want.isnan()), some
        assert torch.equal(got.nan_to_num(9.0), want.nan_to_num(9.0)), some


@pytest.mark.parametrize("n,earlier", [(30, 3001), (500, 0), (512, 1490), (700, 333), (2500, 0)])
def test_heights_of_heads_of_64(n, earlier):
    """Workgroups of 64, 128 and 256 rows: an infinite value and keys that are not numbers reach the
    queries that see them, and change no bit of the others."""
    call = inputs([n], [n + earlier], 32, 8, 64, "f16", seed=n)
    clean = check(call, "f16")
    rest = [d for d in range(64) if d != 5]
    for at in (earlier, earlier + n // 2, earlier + n - 1):
        k, v = call["k"].clone(), call["v"].clone()
        v[at, :, 5] = -float("inf")
        sees = torch.arange(n, device=DEV) + earlier >= at
        got = tv.prompt_attention(**dict(call, k=k, v=v))
        assert (got[sees][..., 5] == -float("inf")).all() and torch.equal(got[..., rest], clean[..., rest])
        assert torch.equal(got[~sees], clean[~sees])
        k[at:] = float("nan")
        got = tv.prompt_attention(**dict(call, k=k, v=v))
        assert torch.isnan(got[sees]).all() and torch.equal(got[~sees], clean[~sees])


def test_large_scores_and_growing_ones():
    """One key holds nearly all of a row's weight; every later key scores higher."""
    check(inputs([300, 20], None, 4, 2, 64, scale_q=40.0))
    check(inputs([300, 20], None, 4, 2, 128, "f16", scale_q=40.0), "f16")
    call = inputs([700], None, 2, 1, 32, "f16")
    q, k = torch.zeros_like(call["q"]), call["k"].clone()
    q[..., 0] = 1.0 / call["scale"]
    k[:, 0, 0] = torch.linspace(0.0, 60.0, 700)
    check(dict(call, q=q, k=k, v=call["v"].clone()), "f16")


def test_other_rows_change_no_bits():
    """A query's bits do not depend on what other queries or sequences ask for."""
    for heads in (4, 32):
        call = inputs([130, 64, 500], None, heads, 4, 64)
        want = tv.prompt_attention(**call)
        q = call["q"].clone()
        q[1::2] *= 30
        q[:, 1::2] *= 30
        assert torch.equal(tv.prompt_attention(**dict(call, q=q))[::2, ::2], want[::2, ::2])
        v = call["v"].clone()
        v[130:194] = float("nan")
        got = tv.prompt_attention(**dict(call, v=v, k=call["k"].clone()))
        assert torch.equal(got[:130], want[:130]) and torch.equal(got[194:], want[194:])


def test_starts_that_decrease_or_leave_the_tensors():
    """They count as the largest before them, and as the nearer end."""
    call = inputs([120], None, 4, 2, 64)
    odd = torch.tensor([-5, 30, 10, -2 ** 31, 70, 2 ** 31 - 1, 100], dtype=torch.int32, device=DEV)
    as_if = torch.tensor([0, 30, 30, 30, 70, 120, 120], dtype=torch.int32, device=DEV)
    want = check(dict(call, q_start=as_if))
    assert torch.equal(tv.prompt_attention(**dict(call, q_start=odd)), want)
    one = torch.tensor([90, 20], dtype=torch.int32, device=DEV)
    out = torch.full((120, 4, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    tv.prompt_attention(**dict(call, q_start=one), out=out)
    assert (out == 3.0).all()


def test_strides_and_a_single_row():
    call = inputs([33, 5], None, 4, 2, 64)
    want = check(call)
    apart = torch.zeros(38, 3, 4, 64, dtype=torch.bfloat16, device=DEV)
    apart[:, 1] = call["q"]
    got = tv.prompt_attention(apart[:, 1], call["k"].contiguous(), call["v"].contiguous(),
                              call["q_start"], call["scale"])
    assert torch.equal(got, want)
    one = inputs([1], None, 4, 2, 64)
    assert torch.equal(tv.prompt_attention(**one), one["v"].repeat_interleave(2, dim=1))


def test_repeated_calls_streams_and_workspaces():
    call = inputs([700, 33, 0, 150], None, 8, 2, 128)
    want = check(call)
    need = tv.tv_prompt_attention_workspace_size(4, 883, 883, 8, 2, 128)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        assert torch.equal(tv.prompt_attention(**call, workspace=ws), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = tv.prompt_attention(**call)
    s.synchronize()
    assert torch.equal(got, want)


def test_two_calls_at_once():
    """On two streams, each with its own workspace."""
    calls = [inputs([900, 300], None, 16, 4, 128, seed=5), inputs([20, 1200, 7], None, 16, 4, 64, seed=6)]
    want = [check(c) for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, c in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                got[i].append(tv.prompt_attention(**c))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert torch.equal(g, want[i])


def test_captured_and_replayed():
    """One capture serves other starts: replays equal eager calls."""
    call = inputs([40, 100, 60], None, 8, 2, 64)
    need = tv.tv_prompt_attention_workspace_size(3, 200, 200, 8, 2, 64)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    out = torch.zeros((200, 8, 64), dtype=torch.bfloat16, device=DEV)
    tv.prompt_attention(**call, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tv.prompt_attention(**call, out=out, workspace=ws)
    for at in ([0, 40, 140, 200], [0, 0, 1, 200], [0, 150, 160, 200], [0, 40, 140, 200]):
        call["q_start"].copy_(torch.tensor(at, dtype=torch.int32))
        want = tv.prompt_attention(**call)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), at


def test_no_keys_at_all():
    """Queries without any key are zeros, whatever the sequences."""
    q = torch.randn((90, 4, 64), device=DEV).to(torch.bfloat16)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    for at in ([0, 90], [0, 33, 33, 90]):
        q_start = torch.tensor(at, dtype=torch.int32, device=DEV)
        got = tv.prompt_attention(q, none, none, q_start, 0.125, k_start=torch.zeros_like(q_start))
        assert not got.any()


def test_first_launch_by_a_graph():
    """The kernel's stack is the runtime's, reserved at a stream's first launch of it: a process whose
    first launch is a graph's replay, on the path that uses the stack, too."""
    code = '''
import torch, paper_2505_12398_amd as tv
g = torch.Generator(device="cuda").manual_seed(1)
qkv = torch.randn((900, 12, 128), generator=g, device="cuda").to(torch.bfloat16)
q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
v[500, :, 7] = float("inf")
at = torch.tensor([0, 900], dtype=torch.int32, device="cuda")
out = torch.zeros((900, 8, 128), dtype=torch.bfloat16, device="cuda")
ws = torch.empty(tv.tv_prompt_attention_workspace_size(1, 900, 900, 8, 2, 128), dtype=torch.uint8, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    tv.prompt_attention(q, k, v, at, 0.09, out=out, workspace=ws)
got = []
for _ in range(3):
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    got.append(out.clone())
want = tv.prompt_attention(q, k, v, at, 0.09)
assert bool((want[500:, :, 7] == float("inf")).all()) and bool(want[:500].isfinite().all())
assert all(torch.equal(x, want) for x in got)
print("equal")
'''
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=100)
    assert run.returncode == 0 and "equal" in run.stdout, run.stderr[-2000:]


def test_offsets_beyond_32_bits():
    """Keys whose rows lie up to 5 GB into their tensor, queries and outputs too."""
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    rows, wide = 40000, 1024
    kv = torch.zeros((rows, wide, 64), dtype=torch.bfloat16, device=DEV)        # 5.2 GB
    g = torch.Generator(device=DEV).manual_seed(2)
    n = 130
    near = torch.randn((n, wide, 64), generator=g, device=DEV).to(torch.bfloat16)
    kv[rows - n:] = near
    at = torch.tensor([rows - n, rows], dtype=torch.int32, device=DEV)
    # (another count of queries may sum in another order: to the bounds, not to the bit)
    for q, k, v in ((slice(0, 8), slice(8, 10), slice(1022, 1024)),
                    (slice(0, 1024), slice(0, 256), slice(256, 512))):
        far = tv.prompt_attention(kv[:, q], kv[:, k], kv[:, v], at, 0.125)
        check(dict(q=near[:, q], k=near[:, k], v=near[:, v], q_start=at - (rows - n), scale=0.125),
              out=far[rows - n:])
