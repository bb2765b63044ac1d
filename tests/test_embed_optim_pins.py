"""Pins for the oracles of the embedding and of 8-bit moments (torch, closed forms, differences), and the refusals of
the C entry points: none of these needs a GPU."""
import copy
import ctypes
import pickle

import numpy as np
import pytest
import torch

from oracle import adamw_oracle as A
from oracle import embedding_oracle as E
from oracle import state8_oracle as S
from paper_2601_02609_amd import binding, build


@pytest.fixture(scope="module")
def L():
    if not build.is_built():
        build.build(verbose=False)
    return binding.lib()


# ------------------------------------------------------------------ embedding
def test_embedding_against_torch_and_autograd():
    rng = np.random.default_rng(0)
    V, D = 11, 6
    w = rng.standard_normal((V, D))
    t = np.array([3, 0, 10, 3, 3, -100, 7, 0])
    dy = rng.standard_normal((len(t), D))
    wt = torch.from_numpy(w).requires_grad_(True)
    ok = t != -100
    y = torch.nn.functional.embedding(torch.from_numpy(t[ok]), wt) * 1.7
    y.backward(torch.from_numpy(dy[ok]))
    out = E.forward(w, t, -100, 1.7)
    assert np.allclose(out[ok], y.detach().numpy(), rtol=1e-15) and not out[~ok].any()
    dw0 = rng.standard_normal((V, D))
    assert np.allclose(E.backward(dy, t, V, -100, 1.7)[0], wt.grad.numpy(), rtol=1e-14)
    assert np.allclose(E.backward(dy, t, V, -100, 1.7, dw0)[0], wt.grad.numpy() + dw0, rtol=1e-14)


def test_embedding_gradient_against_differences():
    rng = np.random.default_rng(1)
    w, t = rng.standard_normal((4, 3)), np.array([1, 1, 9, 2, 0, -1])
    dy = rng.standard_normal((6, 3))
    dw, _ = E.backward(dy, t, 4, -1, 0.5)
    for v in range(4):
        for j in range(3):
            hi, lo = w.copy(), w.copy()
            hi[v, j] += 1e-4
            lo[v, j] -= 1e-4
            num = ((E.forward(hi, t, -1, 0.5) - E.forward(lo, t, -1, 0.5)) * dy).sum() / 2e-4
            assert abs(num - dw[v, j]) <= 1e-9


def test_tokens_that_take_no_part():
    assert E.takes_part([0, 3, 4, -1, -100, 2 ** 31 - 1, 2], 4, 2).tolist() == [True, True, False, False, False, False, False]


# ------------------------------------------------------------------ 8-bit moments
def test_first_moment_codes_are_e4m3():
    ref = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(S.decode(np.arange(256), [127, 127], S.M), ref, equal_nan=True)


def test_second_moment_codes():
    r = S.decode(np.arange(256), [127, 127], S.R)
    assert r[0] == 0.0 and r[1] == 2.0 ** -10 and r[16] == 2.0 ** -6 and r[254] == 480.0 and np.isnan(r[255])
    assert (np.diff(r[:255]) > 0).all() and (r[17:255] / r[16:254] <= 1 + 2.0 ** -4).all()


@pytest.mark.parametrize("bits", [S.M, S.R])
def test_codes_come_back_from_their_values(bits):
    """Whatever the random numbers: a value that has a code in its block's scale keeps it."""
    rng = np.random.default_rng(2)
    for s in (27, 100, 127, 200):
        codes = rng.integers(0, 127 if bits == S.M else 255, 128).astype(np.uint8)
        codes[5] = 0x7E if bits == S.M else 0xFE                            # the largest fixes the scale
        if bits == S.M:
            codes |= (rng.integers(0, 2, 128) << 7).astype(np.uint8)
            codes[codes == 128] = 0
        got, scale = S.encode(S.decode(codes, [s], bits), rng.random(128), bits)
        assert np.array_equal(got, codes) and scale[0] == s


@pytest.mark.parametrize("bits", [S.M, S.R])
def test_rounding_is_unbiased_and_within_a_step(bits):
    rng = np.random.default_rng(3)
    x = np.abs(rng.standard_normal(128)) * np.exp(rng.uniform(-6, 0, 128)) * 1e-3
    got = []
    for k in range(256):
        u = np.full(128, (k + 0.5) / 256)
        codes, scale = S.encode(x, u, bits)
        got.append(S.decode(codes, scale, bits))
    got = np.array(got)
    # two codes are at most 2^-bits of the value apart, below 2^-6 of the scale 2^(-6 - bits) of it
    gap = np.maximum(x * 2.0 ** -bits, 2.0 ** (int(scale[0]) - 127 - 6 - bits))
    assert (np.abs(got - x) < gap).all()
    assert (np.abs(got.mean(0) - x) <= gap / 256).all()
    assert (got.max(0) > got.min(0)).mean() > 0.9


def test_short_block_zeros_and_values_without_a_code():
    x = np.array([0.0, 1e-3, -2e-3, np.inf, np.nan, -np.inf] + [0.0] * 130)
    u = np.full(len(x), 0.999)
    codes, scales = S.encode(x, u, S.M)
    assert codes[3] == 0x7F and codes[4] == 0x7F and codes[5] == 0x7F and codes[0] == 0 and scales[1] == 127
    assert np.isfinite(S.decode(codes, scales, S.M)[[0, 1, 2]]).all()
    codes, scales = S.encode(np.array([1.0, 1e-30, 0.0]), np.zeros(3), S.R)
    assert codes[1] == 1 and codes[2] == 0                                  # a root above 0 stays above 0


def test_random_numbers_are_uniform_and_new_each_step():
    a = [S.dither(1 << 15, 7, t) for t in (1, 2, 3)]
    for um, ur in a:
        for u in (um, ur):
            assert abs(u.mean() - 0.5) <= 5 * np.sqrt(1 / 12 / len(u)) and u.min() >= 0.0 and u.max() < 1.0
        assert abs(np.corrcoef(um, ur)[0, 1]) <= 5 / np.sqrt(len(um))
        assert abs(np.corrcoef(um[1:], um[:-1])[0, 1]) <= 5 / np.sqrt(len(um))
    assert abs(np.corrcoef(a[0][0], a[1][0])[0, 1]) <= 5 / np.sqrt(1 << 15)
    assert not np.array_equal(S.dither(64, 7, 1)[0], S.dither(64, 8, 1)[0])
    whole, part = S.dither(100, 7, 1)[0], S.dither(40, 7, 1, first=60)[0]
    assert np.array_equal(whole[60:], part)


def test_second_moment_follows_a_beta_near_one():
    """The mean over a block of v after 200 steps of a constant gradient is the 32-bit one's within a few percent;
    rounded to nearest it stops growing after a few steps (the reason for the random rounding)."""
    hp = dict(lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)
    g = np.full(128, 0.01)
    zero = (np.zeros(128, np.uint8), np.zeros(1, np.uint8), np.zeros(128, np.uint8), np.zeros(1, np.uint8))
    state, p, m, v = zero, np.zeros(128), np.zeros(128), np.zeros(128)
    near = np.zeros(128)
    for t in range(1, 201):
        _, state, _, _ = S.step(p, g, state, t, 5, **hp)
        _, m, v = A.adamw_step(p, g, m, v, t, **hp)
        near = 0.999 * near + 0.001 * g * g
        near = S.decode(*S.encode(np.sqrt(near), np.full(128, 0.5), S.R), S.R) ** 2
    got = (S.decode(state[2], state[3], S.R) ** 2).mean()
    assert abs(got / v[0] - 1.0) <= 0.05, got / v[0]
    assert near[0] / v[0] <= 0.3


def test_step8_is_adamw_on_what_the_codes_stand_for():
    rng = np.random.default_rng(4)
    n = 300
    p, g = rng.standard_normal(n), rng.standard_normal(n) * 0.01
    m, r = rng.standard_normal(n) * 0.01, np.abs(rng.standard_normal(n)) * 0.01
    state = (*S.encode(m, np.full(n, 0.5), S.M), *S.encode(r, np.full(n, 0.5), S.R))
    got = S.step(p, g, state, 9, 1, 1e-3, 0.9, 0.99, 1e-8, 0.1, clip=0.5)
    want = A.adamw_step(p, g, S.decode(state[0], state[1], S.M), S.decode(state[2], state[3], S.R) ** 2, 9,
                        1e-3, 0.9, 0.99, 1e-8, 0.1, clip=0.5)
    for a, b in zip((got[0], got[2], got[3]), want):
        assert np.allclose(a, b, rtol=1e-13, atol=0)


# ------------------------------------------------------------------ refusals (nothing is enqueued)
P = 1 << 20                                                                 # a well aligned address that nothing looks at


@pytest.mark.parametrize("change,code", [
    (dict(tokens=None), -1), (dict(weight=None), -1), (dict(out=None), -1), (dict(N=0), -1), (dict(N=-3), -1), (dict(D=0), -1),
    (dict(V=0), -1), (dict(D=12), -2), (dict(D=65544), -2), (dict(V=(1 << 24) + 1), -2), (dict(N=1 << 31), -2),
    (dict(weight=P + 8), -1), (dict(out=P + 2), -1), (dict(tokens=P + 2), -1), (dict(status=P + 1), -1)])
def test_embedding_forward_refuses(L, change, code):
    a = dict(tokens=P, weight=P, N=4, D=64, V=100, ignore=-100, scale=1.0, out=P, status=None) | change
    assert L.cce_embedding_forward(a["tokens"], a["weight"], a["N"], a["D"], a["V"], a["ignore"], a["scale"], a["out"], a["status"], None) == code


@pytest.mark.parametrize("change,code", [
    (dict(tokens=None), -1), (dict(d_out=None), -1), (dict(dW=None), -1), (dict(workspace=None), -1), (dict(N=0), -1), (dict(D=-8), -1),
    (dict(V=-1), -1), (dict(D=20), -2), (dict(V=(1 << 24) + 1), -2), (dict(N=1 << 31), -2), (dict(d_out=P + 4), -1), (dict(dW=P + 4), -1),
    (dict(tokens=P + 1), -1), (dict(status=P + 2), -1), (dict(workspace=P + 128), -1), (dict(bytes=0), -1)])
def test_embedding_backward_refuses(L, change, code):
    need = L.cce_embedding_workspace_bytes(4, 64, 100)
    a = dict(tokens=P, d_out=P, N=4, D=64, V=100, ignore=-100, scale=1.0, dW=P, acc=0, status=None, workspace=P, bytes=need) | change
    assert L.cce_embedding_backward(a["tokens"], a["d_out"], a["N"], a["D"], a["V"], a["ignore"], a["scale"], a["dW"], a["acc"], a["status"],
                                    a["workspace"], a["bytes"], None) == code
    if change == dict(bytes=0):
        assert L.cce_embedding_backward(P, P, 4, 64, 100, -100, 1.0, P, 0, None, P, need - 1, None) == -1


def test_embedding_workspace_sizes(L):
    assert L.cce_embedding_workspace_bytes(0, 64, 100) == 0 and L.cce_embedding_workspace_bytes(4, 20, 100) == 0
    for D, V in ((64, 1000), (896, 151936), (8, 3), (8192, 50)):
        ask = [L.cce_embedding_workspace_bytes(n, D, V) for n in (1, 2, 63, 64, 257, 1000, 4097, 8192, 32768, 100000, 1 << 20)]
        assert ask == sorted(ask) and ask[0] > 0, (D, V, ask)


def _entry(**change):
    a = dict(param=P, param_bf16=None, grad=P, m=P, v=P, m_scale=None, v_scale=None, n=100, lr_scale=1.0, weight_decay=0.0,
             grad_bf16=0, state8=0) | change
    return (binding._OptimTensor * 1)(binding._OptimTensor(**a))


def _step(L, entry, **change):
    a = dict(count=1, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, clip=None) | change
    return L.cce_adamw_multi_step(entry, a["count"], a["lr"], a["beta1"], a["beta2"], a["eps"], a["step"], a["clip"], 0, None)


@pytest.mark.parametrize("entry,call,code", [
    (dict(param=None), {}, -1), (dict(grad=None), {}, -1), (dict(m=None), {}, -1), (dict(v=None), {}, -1), (dict(n=-1), {}, -1),
    (dict(n=(1 << 34) + 1), {}, -2), (dict(param=P + 4), {}, -1), (dict(param_bf16=P + 8), {}, -1), (dict(grad=P + 2), {}, -1),
    (dict(m=P + 8), {}, -1), (dict(v=P + 4), {}, -1), (dict(state8=1), {}, -1), (dict(state8=1, m_scale=P), {}, -1), (dict(state8=2), {}, -1),
    (dict(grad_bf16=2), {}, -1), (dict(lr_scale=-1.0), {}, -1), (dict(weight_decay=float("nan")), {}, -1),
    ({}, dict(count=0), -1), ({}, dict(step=0), -1), ({}, dict(beta1=1.0), -1), ({}, dict(beta2=-0.1), -1), ({}, dict(eps=-1.0), -1),
    ({}, dict(lr=float("nan")), -1), ({}, dict(clip=P + 2), -1)])
def test_adamw_multi_refuses(L, entry, call, code):
    assert _step(L, _entry(**entry), **call) == code


def test_adamw_multi_refuses_no_list(L):
    assert _step(L, None) == -1


@pytest.mark.parametrize("entry,call,code", [
    (dict(grad=None), {}, -1), (dict(n=-1), {}, -1), (dict(n=(1 << 34) + 1), {}, -2), (dict(grad=P + 4), {}, -1), (dict(grad_bf16=-1), {}, -1),
    ({}, dict(sumsq=None), -1), ({}, dict(sumsq=P + 4), -1), ({}, dict(ws=None), -1), ({}, dict(ws=P + 8), -1), ({}, dict(bytes=8191), -1),
    ({}, dict(count=0), -1), ({}, dict(clip=P, max_norm=0.0), -1), ({}, dict(clip=P, max_norm=float("nan")), -1), ({}, dict(clip=P, eps=-1.0), -1),
    ({}, dict(clip=P + 1), -1)])
def test_sumsq_multi_refuses(L, entry, call, code):
    a = dict(count=1, sumsq=P, max_norm=1.0, eps=1e-6, clip=None, ws=P, bytes=L.cce_sumsq_multi_workspace_bytes(1)) | call
    assert L.cce_grad_sumsq_multi(_entry(**entry), a["count"], a["sumsq"], 0, a["max_norm"], a["eps"], a["clip"], a["ws"], a["bytes"], None) == code


@pytest.mark.parametrize("sizes,too_many", [([1 << 33], False), ([(1 << 33) + 1], True), ([1 << 33] * 128, False), ([1 << 33] * 128 + [1], True),
                                            ([(1 << 33) - 1] * 128 + [128], False), ([1] * 5000 + [0], False)])
def test_limits_of_a_list(L, sizes, too_many):
    """A tensor of 2^33 values and 2^40 in all are the most that a list holds.  The calls are refused in either case: what is
    within the limits for the argument that is missing."""
    entries = (binding._OptimTensor * len(sizes))(*[binding._OptimTensor(param=P, grad=P, m=None, v=P, n=n, lr_scale=1.0) for n in sizes])
    code = -2 if too_many else -1
    need = L.cce_sumsq_multi_workspace_bytes(len(sizes))
    assert L.cce_grad_sumsq_multi(entries, len(sizes), None, 0, 1.0, 1e-6, None, P, need, None) == code
    assert L.cce_adamw_multi_step(entries, len(sizes), 1e-3, 0.9, 0.99, 1e-8, 1, None, 0, None) == code


def test_state8_read_refuses(L):
    for codes, scales, n, second, out in ((None, P, 5, 0, P), (P, None, 5, 0, P), (P, P, 0, 0, P), (P, P, 5, 2, P), (P + 4, P, 5, 0, P), (P, P, 5, 0, P + 8)):
        assert L.cce_adamw_state8_read(codes, scales, n, second, out, None) == -1


def test_binding_refuses_host_tensors(L):
    with pytest.raises(ValueError):
        binding.cce_embedding_forward(torch.zeros(3, dtype=torch.int32), torch.zeros(5, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        binding.OptimTensors([torch.zeros(3)])
    with pytest.raises(ValueError):
        binding.OptimTensors([])
    with pytest.raises(ValueError):
        binding.cce_adamw_state8_read(torch.zeros(3, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8))
    assert ctypes.sizeof(binding._OptimTensor) == 80


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, pickle.dumps])
def test_lists_are_not_copied(how):
    """A copy would give the library the address of the original's table, which names the original's tensors and may be gone."""
    tensors = object.__new__(binding.OptimTensors)
    tensors._table = np.zeros(1, dtype=np.dtype(binding._OptimTensor))
    tensors._address = tensors._table.ctypes.data
    with pytest.raises(TypeError, match="OptimTensors"):
        how(tensors)


class _Tensor:
    """What a list asks of a tensor, without a device."""
    address = 1 << 20

    def __init__(self, dtype, n):
        self.dtype, self.n, self.device, self.is_cuda, self.on = dtype, n, torch.device("cuda:0"), True, []
        self.at, _Tensor.address = _Tensor.address, _Tensor.address + (4 * n + 255) // 256 * 256

    numel = lambda self: self.n
    is_contiguous = lambda self: True
    data_ptr = lambda self: self.at
    record_stream = lambda self, stream: self.on.append(stream.cuda_stream)


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.mark.parametrize("state8", [False, True])
def test_tensors_of_a_list_are_kept_for_the_stream_that_reads_them(monkeypatch, state8):
    """A call on a stream of the caller's returns before its kernels have run: memory of the list, of gradients that
    set_grads replaces above all, must not be handed out again until that stream has done with it."""
    monkeypatch.setattr(binding, "_call", lambda *args: None)
    monkeypatch.setattr(binding, "_new", lambda *args: torch.zeros(1))
    f32, moment = torch.float32, torch.uint8 if state8 else torch.float32
    new = lambda dtype, *sizes: [_Tensor(dtype, n) for n in sizes]
    grads, copies = new(f32, 300, 0), [_Tensor(torch.bfloat16, 300), None]
    rest = [new(f32, 300, 0), new(moment, 300, 0), new(moment, 300, 0)]
    scales = [new(torch.uint8, 3, 0), new(torch.uint8, 3, 0)] if state8 else [None, None]
    T = binding.OptimTensors(grads, *rest, params_bf16=copies, m_scales=scales[0], v_scales=scales[1])
    a, b = _Stream(11), _Stream(12)
    step = lambda stream: binding.cce_adamw_multi_step(T, 1, lr=1e-3, stream=stream)
    norm = lambda stream: binding.cce_grad_sumsq_multi(T, stream=stream)
    step(None)                                                              # the current stream: torch's own rule
    assert all(t.on == [] for t in grads)
    for _ in range(2):
        step(a)
    everything = [t for part in (grads, copies, *rest, *(x for x in scales if x)) for t in part if t is not None]
    assert all(t.on == [11] for t in everything)
    later = new(torch.bfloat16, 300, 0)
    T.set_grads(later)
    step(a)
    assert all(t.on == [11] for t in later)
    norm(b)
    assert all(t.on == [11, 12] for t in later)
    step(b)
    assert all(t.on == [11, 12] for t in rest[0]) and all(t.on == [11] for t in grads)
