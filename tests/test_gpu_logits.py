"""tv_process_logits against the plain 64-bit form (needs an MI355X)."""

import math

import numpy as np
import pytest
import torch

import paper_2505_12398_amd as tv
from oracle import decoding as D

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    tv.load_library()
    yield


def case(batch, n1, V, dtype=torch.bfloat16, hist=50, bias=0, masks=0, seed=0, few=None, chain=False):
    """Host (numpy) and device inputs. ``few``: token ids below that, so that they repeat."""
    rng = np.random.default_rng([seed, batch, n1, V])
    few = few or V
    z = torch.tensor(rng.normal(0, 4, (batch, n1, V))).to(dtype)
    par = np.full((batch, n1), -1, np.int32)
    for i in range(1, n1):
        par[:, i] = i - 1 if chain else rng.integers(max(0, i - 4), i, batch)
    h = dict(logits=z, parents=par, tokens=rng.integers(0, few, (batch, n1)),
             history=rng.integers(0, few, (batch, hist)),
             history_len=rng.integers(0, hist + 1, batch),
             prompt_len=rng.integers(0, hist + 1, batch),
             repetition=rng.uniform(0.7, 1.6, batch), presence=rng.uniform(-1, 1, batch),
             frequency=rng.uniform(-1, 1, batch))
    if bias:
        h["bias_tokens"] = rng.integers(-2, few, (batch, bias))
        h["bias_values"] = np.where(rng.random((batch, bias)) < 0.2, -np.inf,
                                    rng.normal(0, 3, (batch, bias)))
    if masks:
        h["masks"] = rng.integers(-2 ** 31, 2 ** 31, (masks, (V + 31) // 32))
        h["mask_index"] = rng.integers(-1, masks, (batch, n1))
    real = ("repetition", "presence", "frequency", "bias_values")
    call = {k: torch.as_tensor(np.asarray(v), device=DEV).to(
        torch.float32 if k in real else torch.int32) for k, v in h.items() if k != "logits"}
    call["logits"] = z.to(DEV)
    for k in real:
        if k in h:
            h[k] = np.asarray(h[k], np.float32).astype(np.float64)
    h["logits"] = z.double().numpy()
    return h, call


def expected(h, b):
    V = h["logits"].shape[-1]
    hist = h.get("history")
    n = min(max(int(h["history_len"][b]), 0), hist.shape[1]) if hist is not None else 0
    p = min(max(int(h["prompt_len"][b]), 0), n) if "prompt_len" in h and hist is not None else 0
    allowed = None
    if "mask_index" in h:
        allowed = []
        for m in h["mask_index"][b]:
            if m < 0:
                allowed.append(None)
            elif m >= len(h["masks"]):
                allowed.append(np.zeros(V, bool))
            else:
                w = h["masks"][m].astype(np.int64) & 0xffffffff
                allowed.append(np.array([(w[t // 32] >> (t % 32)) & 1 for t in range(V)], bool))
    biases = list(zip(h["bias_tokens"][b], h["bias_values"][b])) if "bias_tokens" in h else []
    return D.process_logits(h["logits"][b], h.get("parents")[b] if "parents" in h else None,
                            h["tokens"][b] if "tokens" in h else None,
                            hist[b][:n] if hist is not None else [], p,
                            float(h["repetition"][b]) if "repetition" in h else 1.0,
                            float(h["presence"][b]) if "presence" in h else 0.0,
                            float(h["frequency"][b]) if "frequency" in h else 0.0, biases, allowed)


def check(h, call, T=1.0, rows=None, most=0.0, **kw):
    """Logits: one rounding to the type, and in fp32 one each of the penalised logit, frequency
    times count, the sum of the penalties, that less the bias and the difference, each of at
    most ``size``. Statistics: of the logits as they came out."""
    out, mx, sm = tv.process_logits(temperature=T, **call, **kw)
    B, n1, V = out.shape
    first, count = rows or (0, n1)
    half = torch.finfo(out.dtype).eps / 2
    z = out.double().cpu().numpy()
    for b in range(B):
        want = expected(h, b)
        with np.errstate(invalid="ignore"):
            fine = np.isfinite(want)
            big = np.abs(np.where(fine, want, 0)) + 2 * np.abs(
                np.where(fine, h["logits"][b], 0)) * 1.6 + 12 + most
        r = slice(first, first + count)
        assert np.array_equal(z[b, r][~fine[r]], want[r][~fine[r]], equal_nan=True)
        err = np.abs(np.where(fine, z[b], 0) - np.where(fine, want, 0))
        tol = half * np.abs(np.where(fine, want, 0)) + 6 * 2.0 ** -24 * big
        assert (err[r] <= tol[r]).all(), float((err / tol)[r].max())
        if mx is None:
            continue
        top = z[b, r].max(axis=1)
        assert np.array_equal(mx[b, r].cpu().numpy().astype(np.float64), top, equal_nan=True)
        got = sm[b, r].cpu().numpy()
        for i in range(count):
            if not np.isfinite(top[i]):
                continue
            total = np.exp((z[b, first + i] - top[i]) / float(np.float32(T))).sum()
            # fp32 terms: exponents of up to (range of the row) k, rounded thrice; hardware exp2
            assert abs(got[i] - total) <= 2e-6 * total, (b, i, got[i], total)
    return out, mx, sm


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [2, 7, 8, 31, 257, 8191, 8192, 8193, 20003])
@pytest.mark.parametrize("n1", [1, 6])
def test_sizes(dtype, V, n1):
    """Around a thread's eight tokens and a workgroup's 8192; rows off the 16-byte grid."""
    h, call = case(3, n1, V, dtype, bias=5, masks=3, few=min(V, 40))
    check(h, call, T=0.7)


def test_rows_of_many_trees_and_few():
    for batch, n1 in ((1, 65), (40, 9)):
        h, call = case(batch, n1, 1000, hist=300, few=200, seed=batch)
        check(h, call)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tokens_that_repeat_on_the_path(dtype):
    """A long chain over few tokens: counts that grow along the path, at every place."""
    h, call = case(2, 200, 64, dtype, hist=30, bias=10, few=5, chain=True)
    h["frequency"] *= 0.01
    call["frequency"] *= 0.01
    h["frequency"] = call["frequency"].double().cpu().numpy()
    check(h, call, most=8.0)


def test_links_and_tokens_that_are_none():
    h, call = case(2, 6, 100, few=20)
    for name, value in (("parents", [[-1, 0, 9, 2, -3, 4]] * 2),
                        ("tokens", [[3, -1, 5, 5, 100, 1 << 30]] * 2)):
        h[name] = np.array(value)
        call[name] = torch.tensor(value, dtype=torch.int32, device=DEV)
    h["history"][:, ::3] = -5
    h["history"][:, 1::3] = 100
    call["history"] = torch.as_tensor(h["history"], device=DEV).to(torch.int32)
    check(h, call)


def test_each_part_alone():
    """Any of the inputs may be left out; without all of them the logits pass through."""
    h, call = case(3, 5, 300, bias=6, masks=2, few=30)
    groups = (("parents", "tokens"), ("history", "history_len", "prompt_len"), ("prompt_len",),
              ("repetition",), ("presence",), ("frequency",), ("bias_tokens", "bias_values"),
              ("masks", "mask_index"))
    for g in groups:
        less = {k: v for k, v in h.items() if k not in g}
        check(less, {k: v for k, v in call.items() if k not in g})
        only = {k: v for k, v in call.items() if k in g + ("logits", "history", "history_len")}
        check({k: v for k, v in h.items() if k in g + ("logits", "history", "history_len")}, only)
    out, _, _ = tv.process_logits(call["logits"], 1.0)
    assert torch.equal(out, call["logits"])


def test_lengths_beyond_the_history_and_below_zero():
    h, call = case(4, 3, 100, few=30)
    for name, v in (("history_len", [60, -3, 20, 50]), ("prompt_len", [70, 5, -1, 1 << 30])):
        h[name] = np.array(v)
        call[name] = torch.tensor(v, dtype=torch.int32, device=DEV)
    check(h, call)


def test_the_last_of_several_biases_counts():
    h, call = case(1, 2, 50, bias=7)
    h["bias_tokens"][:] = [[4, 4, 9, 4, 9, -1, 50]]
    h["bias_values"][:] = [[1, 2, 3, -np.inf, 0.5, 7, 7]]
    call["bias_tokens"] = torch.as_tensor(h["bias_tokens"], device=DEV).to(torch.int32)
    call["bias_values"] = torch.as_tensor(h["bias_values"], device=DEV).to(torch.float32)
    out, _, _ = check(h, call)
    assert (out[0, :, 4] == -math.inf).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinities_nan_and_masked_rows(dtype):
    """-inf stays, NaN and +inf show in the statistics unless they are masked; a mask that allows
    nothing, and one that there is not, give a row of -inf with maximum -inf and sum 0."""
    h, call = case(1, 7, 90, dtype, hist=1, masks=3, few=80)
    z, m = call["logits"], call["masks"]
    m[0], m[1] = -1, 0
    m[2] = -1
    m[2, 0] = ~(1 << 5)
    idx = torch.tensor([[-1, 1, 3, 0, 0, 2, 2]], dtype=torch.int32, device=DEV)
    call["mask_index"] = idx
    z[0, 0, 10:20] = -math.inf
    z[0, 3, 7] = math.nan
    z[0, 4, 7] = math.inf
    z[0, 5, 5] = math.nan
    z[0, 6, 5] = math.inf
    for name in ("history", "parents", "tokens", "history_len", "prompt_len"):
        call.pop(name)
    call.update(repetition=None, presence=None, frequency=None)
    out, mx, sm = tv.process_logits(temperature=1.0, **call)
    assert torch.equal(out[0, 0], z[0, 0])
    assert (out[0, 1:3] == -math.inf).all()
    assert mx[0, 1:3].tolist() == [-math.inf] * 2 and sm[0, 1:3].tolist() == [0.0] * 2
    assert not math.isfinite(sm[0, 3]) and not math.isfinite(sm[0, 4])
    assert torch.isnan(out[0, 3, 7]) and out[0, 4, 7] == math.inf
    for i in (0, 5, 6):
        row = out[0, i].double()
        assert mx[0, i].double() == row.max()
        total = float((row - row.max()).exp().sum())
        assert abs(float(sm[0, i]) - total) <= 2e-6 * total


def test_penalised_infinities():
    """Penalties leave infinities infinite, and NaN NaN."""
    z = torch.tensor([[[math.inf, -math.inf, math.nan, 3.0e38, -3.0e38, 0.0]]], device=DEV)
    hist = torch.arange(6, dtype=torch.int32, device=DEV)[None]
    n = torch.tensor([6], dtype=torch.int32, device=DEV)
    out, _, _ = tv.process_logits(z, 1.0, history=hist, history_len=n,
                                  repetition=torch.tensor([2.0], device=DEV))
    got = out[0, 0].tolist()
    assert got[:2] == [math.inf, -math.inf] and math.isnan(got[2])
    assert got[3] == float(z[0, 0, 3]) / 2 and got[4:] == [-math.inf, 0.0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place_and_some_nodes(dtype):
    """In place; a level of nodes leaves the others as they were."""
    h, call = case(3, 8, 500, dtype, bias=4, masks=2, few=60)
    want, mx, sm = check(h, call)
    z = call["logits"].clone()
    before = z.clone()
    for first, count in ((0, 1), (1, 3), (4, 4)):
        out, m, s = tv.process_logits(temperature=1.0, **dict(call, logits=z), out=z,
                                      nodes=(first, count))
        r = slice(first, first + count)
        assert out is z and torch.equal(z[:, r], want[:, r])
        assert torch.equal(z[:, first + count:], before[:, first + count:])
        assert torch.equal(m[:, r], mx[:, r]) and torch.equal(s[:, r], sm[:, r])
    out, m, s = tv.process_logits(temperature=1.0, **call, want_stats=False)
    assert torch.equal(out, want) and m is None and s is None


def test_unaligned_tensors():
    """Logits and result that start off the 16-byte grid, differently."""
    h, call = case(2, 3, 1001, few=50, masks=2)
    n = call["logits"].numel()
    a = torch.empty(n + 8, dtype=torch.bfloat16, device=DEV)
    o = torch.full((n + 8,), 5.0, dtype=torch.bfloat16, device=DEV)
    z = a[1:1 + n].view(2, 3, 1001)
    z.copy_(call["logits"])
    check(h, dict(call, logits=z), out=o[3:3 + n].view(2, 3, 1001))
    assert (o[:3] == 5.0).all() and (o[3 + n:] == 5.0).all()


@pytest.mark.parametrize("T", [1e-3, 0.05, 1.0, 100.0])
def test_statistics_at_temperatures(T):
    """In place of 2e-6: exponents x = (z - max)/T of up to `span` have errors of 2^-22 |x| where
    their terms still count (x exp(-x) < 1/e for each of the V terms)."""
    h, call = case(2, 3, 3000, torch.float32)
    out, mx, sm = tv.process_logits(temperature=T, **call)
    z = out.double()
    t32 = float(np.float32(T))
    x = (z - z.amax(-1, keepdim=True)) / t32
    total = x.exp().sum(-1)
    frame = (z.abs().amax(-1) / t32)                    # the frame -max k is rounded to fp32
    slack = (x.abs() * x.exp()).sum(-1) * 2 ** -22 + total * (2 ** -20 + frame * 0)
    assert torch.equal(mx, out.float().amax(-1))
    assert ((sm - total).abs() <= slack + total * frame * 2 ** -23).all()


def test_long_history():
    """More occurrences of a token than 16 bits count."""
    hist = torch.full((1, 70000), 3, dtype=torch.int32, device=DEV)
    hist[0, :1000] = 5
    z = torch.zeros((1, 1, 10), device=DEV)
    out, _, _ = tv.process_logits(z, 1.0, history=hist,
                                  history_len=torch.tensor([70000], dtype=torch.int32, device=DEV),
                                  prompt_len=torch.tensor([500], dtype=torch.int32, device=DEV),
                                  frequency=torch.tensor([1.0], device=DEV),
                                  presence=torch.tensor([0.5], device=DEV))
    assert out[0, 0].tolist() == [0, 0, 0, -69000.5, 0, -500.5, 0, 0, 0, 0]


def test_captured_and_replayed():
    h, call = case(3, 5, 2000, bias=3, masks=2, few=100)
    _, other = case(3, 5, 2000, bias=3, masks=2, few=100, seed=9)
    out = torch.empty_like(call["logits"])
    ws = torch.empty(tv.tv_process_logits_workspace_size(3, 5, 2000), dtype=torch.uint8, device=DEV)
    tv.process_logits(temperature=1.0, **call, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, mx, sm = tv.process_logits(temperature=1.0, **call, out=out, workspace=ws)
    first = {k: v.clone() for k, v in call.items()}
    for k in range(4):
        src = first if k % 2 == 0 else other
        for name in call:
            call[name].copy_(src[name])
        want = tv.process_logits(temperature=1.0, **call)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((out, mx, sm), want):
            assert torch.equal(got, w), k


def test_statistics_feed_the_verifier():
    """tv_verify_stats on the processed logits of both models equals tv_verify on them."""
    import parity
    import workloads as W
    bt = W.make_batch(5, step=3, device=DEV, mode=W.WITHOUT_REPLACEMENT, batch=16, vocab=20011)
    kw = dict(parents=bt["parents"], tokens=bt["tokens"],
              history=torch.randint(0, 20011, (16, 500), dtype=torch.int32, device=DEV),
              history_len=torch.full((16,), 400, dtype=torch.int32, device=DEV),
              prompt_len=torch.full((16,), 100, dtype=torch.int32, device=DEV),
              repetition=torch.full((16,), 1.2, device=DEV),
              presence=torch.full((16,), 0.3, device=DEV),
              frequency=torch.full((16,), 0.2, device=DEV))
    T = bt["temperature"]
    target, tm, ts = tv.process_logits(bt["target"], T, **kw)
    draft, dm, ds = tv.process_logits(bt["draft"], T, **kw)
    args = (bt["parents"], bt["tokens"], target, draft, T, bt["uniforms"], bt["mode"])
    a = parity.host_outputs(tv.verify_batch(*args, stats=(tm, ts, dm, ds)))
    rep = parity.check(dict(bt, target=target, draft=draft), False, gpu=a, label="processed")
    assert not rep.failures, rep.failures[:3]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_penalised_quotients_are_those_of_a_division(dtype):
    """z / repetition for repetitions below and above 1 and down to subnormal ones, at logits up
    to the largest: as the host divides, infinite where that is."""
    rng = np.random.default_rng(4)
    rho = np.array([0.7, 0.999, 1e-3, 1e-20, 1e-37, 1e-40, 3e-45, 1.0, 1.3, 7.0, 1e10, 2e38],
                   np.float32)
    top = torch.finfo(dtype).max
    z = np.concatenate([rng.normal(0, 4, 40), 10.0 ** rng.uniform(-20, 38.4, 40),
                        [3e38, top, top * 0.7, 1e-10, 2.0, 0.0, -0.0]])
    z = torch.tensor(np.repeat(z[None, None], len(rho), 0)).to(dtype).to(DEV)
    V = z.shape[-1]
    hist = torch.arange(V, dtype=torch.int32, device=DEV).repeat(len(rho), 1)
    n = torch.full((len(rho),), V, dtype=torch.int32, device=DEV)
    out, mx, _ = tv.process_logits(z, 1.0, history=hist, history_len=n, prompt_len=n,
                                   repetition=torch.tensor(rho, device=DEV))
    x = z.float().cpu().numpy()
    with np.errstate(over="ignore"):
        want = np.where(x > 0, x / rho[:, None, None], x * rho[:, None, None]).astype(np.float32)
    want = torch.tensor(want).to(dtype)
    # (quotients that are no normal numbers are not claimed to the bit)
    small = want.double().abs() < 2.0 ** -126
    got = out.cpu()
    assert torch.equal(got[~small], want[~small])
    assert (got.double()[small] - want.double()[small]).abs().max() <= 2.0 ** -126 * \
        torch.finfo(dtype).eps
    assert torch.equal(mx.cpu(), want.float().amax(-1))


def test_penalised_quotients_on_the_path():
    """The same for tokens that a node's path has."""
    z = torch.tensor([[[3e38, 3e38, 1.0, 1e-10]] * 2] * 2, device=DEV)
    par = torch.tensor([[-1, 0]] * 2, dtype=torch.int32, device=DEV)
    rho = torch.tensor([0.7, 1e-40], device=DEV)
    for t in range(4):
        tok = torch.tensor([[0, t]] * 2, dtype=torch.int32, device=DEV)
        out, _, _ = tv.process_logits(z, 1.0, parents=par, tokens=tok, repetition=rho)
        with np.errstate(over="ignore"):
            want = z.cpu().numpy().copy()
            want[:, 1, t] = want[:, 1, t] / rho.cpu().numpy()
        assert np.array_equal(out.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1.0, 0.05, 1e-3, 1e3])
@pytest.mark.parametrize("low", [-1e9, -3e10, -1e20, -1e30, -1e37, -3.3e38, None])
def test_statistics_of_rows_masked_with_low_values(dtype, T, low):
    """Masks by a large negative number, down to the type's lowest: on part of a row, in whole
    wavefronts' and workgroups' parts, in all of it. Terms as in ``check``: exponents of finite
    range here (a masked entry's is below -800 next to one that is not)."""
    V = 20003
    rng = np.random.default_rng(6)
    low = torch.finfo(dtype).min if low is None else low
    z = torch.tensor(rng.normal(0, 1, (1, 8, V)))
    z[0, 0, ::3] = low
    z[0, 1, :9000] = low
    z[0, 2, 5:] = low
    z[0, 3, :-1] = low
    z[0, 4] = low
    z[0, 5] = low
    z[0, 5, 8192:8200] = -math.inf
    z[0, 6] = low
    z[0, 6, 17] = low * 0.5
    z[0, 7, 9000] = -low
    z = z.to(dtype).to(DEV)
    out, mx, sm = tv.process_logits(z, T)
    assert torch.equal(out, z)
    row = z[0].double()
    assert torch.equal(mx[0].double(), row.amax(-1))
    x = (row - row.amax(-1, keepdim=True)) / float(np.float32(T))
    total = x.exp().sum(-1)
    # exponents with errors of 2^-22 |x|; a thread's 32 terms, the wavefront's and an exponential's
    # roundings
    slack = (x.abs() * x.exp()).nan_to_num(0.0).sum(-1) * 2.0 ** -22 + total * 42 * 2.0 ** -24
    assert ((sm[0] - total).abs() <= slack).all(), (sm[0].tolist(), total.tolist())


def test_more_rows_than_one_grid_of_wavefronts():
    """2^26 rows and more of a vocabulary of two."""
    B, n1 = 65537, 1024
    g = torch.Generator(device=DEV).manual_seed(3)
    z = torch.randn((B, n1, 2), generator=g, device=DEV).bfloat16()
    out, mx, sm = tv.process_logits(z, 1.0, want_stats=True)
    assert torch.equal(out, z)
    for part in (slice(0, 100), slice(-100, None), slice(32000, 34000)):
        r = z[part].double()
        assert torch.equal(mx[part].double(), r.amax(-1))
        want = (r - r.amax(-1, keepdim=True)).exp().sum(-1)
        assert ((sm[part] - want).abs() <= 2e-6 * want).all()
    assert bool(((sm > 1.0) & (sm <= 2.0 + 1e-5)).all())


def test_drafted_tokens_of_long_bias_lists():
    """The bias of a drafted token is not looked for in the list row by row: 50000 biases cost a
    call about what 500 cost."""
    B, n1, V = 4, 33, 32000
    z = torch.randn((B, n1, V), device=DEV).bfloat16()
    par = torch.arange(-1, n1 - 1, dtype=torch.int32, device=DEV).repeat(B, 1)
    tok = torch.arange(n1, dtype=torch.int32, device=DEV).repeat(B, 1) * 3
    us = {}
    for n in (500, 50000):
        at = (V - 1 - torch.arange(n, device=DEV) % (V - 200)).int().repeat(B, 1)
        at[:, :300] = torch.arange(300, device=DEV).int()      # drafted tokens at the list's start
        val = torch.randn((B, n), device=DEV)
        kw = dict(parents=par, tokens=tok, bias_tokens=at.contiguous(), bias_values=val,
                  frequency=torch.full((B,), 0.5, device=DEV))
        out, _, _ = tv.process_logits(z, 1.0, **kw)
        last = torch.zeros((B, V), device=DEV)
        for b in range(B):
            keep = {}
            for j, t in enumerate(at[b].tolist()):
                keep[t] = j
            idx = torch.tensor(list(keep.items()), device=DEV)
            last[b, idx[:, 0]] = val[b, idx[:, 1]]
        seen = torch.zeros((B, n1, V), device=DEV)
        for i in range(1, n1):
            seen[:, i:, 3 * i] = 0.5
        want = (z.float() - (seen - last[:, None])).bfloat16()
        assert torch.equal(out, want)
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        torch.cuda.synchronize()
        e[0].record()
        for _ in range(3):
            tv.process_logits(z, 1.0, **kw)
        e[1].record()
        torch.cuda.synchronize()
        us[n] = e[0].elapsed_time(e[1]) / 3 * 1e3
    assert us[50000] < 40 * us[500] + 2000, us
