"""Host-side checks of the operators for batches of many requests: refusals
before any HIP call (fake, aligned, non-null device pointers), workspace sizes,
and the binding's checks of shapes."""
import numpy as np
import pytest

import requests_ref as R


@pytest.fixture(scope="module")
def dl():
    import paper_2606_10932_amd as D
    return D


def _step(dl, ld=8512, M=1, di=4096, N=128, P=64, slots=16, pos=16, n=4, zx=16, ring=16, state=16, y=16, w=16):
    return dl.lib.dfssm_ssm_step_slots(zx, ld, M, di, N, P, slots, pos, n, ring, w, 16, 16, 16, 16, state, y, None)


def test_step_slots_validation(dl):
    assert _step(dl, P=32) == dl.ERR_UNSUPPORTED
    assert _step(dl, N=96) == dl.ERR_UNSUPPORTED
    assert _step(dl, di=4000) == dl.ERR_SHAPE
    assert _step(dl, di=65536 + 64, ld=1 << 20) == dl.ERR_SHAPE
    assert _step(dl, ld=8511) == dl.ERR_SHAPE
    assert _step(dl, ld=(1 << 22) + 1) == dl.ERR_SHAPE
    assert _step(dl, M=-1) == dl.ERR_SHAPE
    assert _step(dl, M=65537) == dl.ERR_SHAPE
    assert _step(dl, n=-1) == dl.ERR_SHAPE
    assert _step(dl, n=1 << 31) == dl.ERR_SHAPE
    assert _step(dl, zx=None) == dl.ERR_NULL
    assert _step(dl, slots=None) == dl.ERR_NULL and "slots" in dl.last_error()
    assert _step(dl, pos=None) == dl.ERR_NULL
    assert _step(dl, ring=None) == dl.ERR_NULL
    assert _step(dl, state=None) == dl.ERR_NULL
    assert _step(dl, slots=18) == dl.ERR_ALIGN
    assert _step(dl, pos=17) == dl.ERR_ALIGN
    assert _step(dl, y=20) == dl.ERR_ALIGN
    assert _step(dl, w=8) == dl.ERR_ALIGN
    assert _step(dl, M=0, zx=None, slots=None) == dl.OK


def _prompt(dl, ld=8512, T=100, S=2, di=4096, N=128, P=64, cu=16, slots=16, pos=16, n=4, zx=16, ring=16, state=16,
            y=16, ws=16, wsb=1 << 40):
    return dl.lib.dfssm_ssm_prompt(zx, ld, T, cu, S, di, N, P, slots, pos, n, ring, 16, 16, 16, 16, 16, state, y, ws,
                                   wsb, None)


def test_step_slots_more_workgroups_than_a_launch_has(dl):
    # 2^14 rows of 1024 heads: 2^24 workgroups of 256 threads
    assert _step(dl, M=1 << 14, di=65536, ld=1 << 20) == dl.ERR_SHAPE and "2^24" in dl.last_error()


def test_prompt_validation(dl):
    assert _prompt(dl, P=128) == dl.ERR_UNSUPPORTED
    assert _prompt(dl, N=32) == dl.ERR_UNSUPPORTED
    assert _prompt(dl, di=0) == dl.ERR_SHAPE
    assert _prompt(dl, ld=8511) == dl.ERR_SHAPE
    assert _prompt(dl, T=-1) == dl.ERR_SHAPE
    assert _prompt(dl, T=(1 << 24) + 1) == dl.ERR_SHAPE
    assert _prompt(dl, S=-1) == dl.ERR_SHAPE
    assert _prompt(dl, S=4097) == dl.ERR_SHAPE
    assert _prompt(dl, n=-1) == dl.ERR_SHAPE
    assert _prompt(dl, slots=None, S=5) == dl.ERR_SHAPE and "slots" in dl.last_error()
    assert _prompt(dl, zx=None) == dl.ERR_NULL
    assert _prompt(dl, cu=None) == dl.ERR_NULL
    assert _prompt(dl, ring=None) == dl.ERR_NULL
    assert _prompt(dl, ws=None) == dl.ERR_NULL
    assert _prompt(dl, cu=18) == dl.ERR_ALIGN
    assert _prompt(dl, slots=21) == dl.ERR_ALIGN
    assert _prompt(dl, pos=22) == dl.ERR_ALIGN
    assert _prompt(dl, state=24) == dl.ERR_ALIGN
    assert _prompt(dl, ws=24) == dl.ERR_ALIGN
    need = dl.ssm_prompt_workspace_bytes(100, 2, 4096)
    assert need > 0 and _prompt(dl, wsb=need - 1) == dl.ERR_WORKSPACE
    assert _prompt(dl, T=0, zx=None, cu=None, ws=None, wsb=0) == dl.OK
    assert _prompt(dl, S=0, zx=None, cu=None, ws=None, wsb=0) == dl.OK
    # sizes outside the limits have no workspace
    for bad in ((-1, 1, 4096), (1, -1, 4096), (1 << 25, 1, 4096), (1, 5000, 4096), (1, 1, 0)):
        assert dl.ssm_prompt_workspace_bytes(*bad) == 0
    assert dl.ssm_prompt_workspace_bytes(1, 1, 64, 96) == 0


@pytest.mark.parametrize("d_inner,N", [(64, 64), (1536, 128), (4096, 128), (5120, 64), (65536, 128)])
def test_prompt_workspace_never_falls(dl, d_inner, N):
    """A workspace for T rows and S sequences serves every smaller call."""
    size = lambda T, S: dl.ssm_prompt_workspace_bytes(T, S, d_inner, N)
    for S in (1, 2, 6, 33, 4096):
        sizes = [size(T, S) for T in range(1, 9000)] + [size(T, S) for T in range(9000, 1 << 24, 99991)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), S
    for T in (1, 64, 383, 384, 3008, 100000):
        sizes = [size(T, S) for S in range(1, 4097)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), T


def _adapt(dl, M=2, K=64, N=8, r=4, n=3, ids=16, A=16, B=16, be=16, y=16, out=16, ws=16, wsb=1 << 20, q=16, s=16, i4=False):
    f = dl.lib.dfssm_lora_adapters_i4 if i4 else dl.lib.dfssm_lora_adapters
    return f(q, s, M, K, N, r, ids, n, A, B, be, y, out, ws, wsb, None)


@pytest.mark.parametrize("i4", [False, True])
def test_adapters_validation(dl, i4):
    f = lambda **kw: _adapt(dl, i4=i4, **kw)
    assert f(K=48) == dl.ERR_SHAPE
    assert f(K=65536 + 32) == dl.ERR_SHAPE
    assert f(M=-1) == dl.ERR_SHAPE
    assert f(N=-1) == dl.ERR_SHAPE
    assert f(N=(1 << 24) + 1) == dl.ERR_SHAPE
    assert f(r=257) == dl.ERR_SHAPE
    assert f(r=-2) == dl.ERR_SHAPE
    assert f(n=-1) == dl.ERR_SHAPE
    assert f(n=1 << 31) == dl.ERR_SHAPE
    for name in ("q", "s", "ids", "A", "B", "be", "y", "out", "ws"):
        assert f(**{name: None}) == dl.ERR_NULL, name
    for name in ("q", "s", "A", "B", "be", "y", "out", "ws"):
        assert f(**{name: 24}) == dl.ERR_ALIGN, name
    assert f(ids=18) == dl.ERR_ALIGN
    need = dl.lora_adapters_workspace_bytes(2, 4)
    assert need > 0 and f(wsb=need - 1) == dl.ERR_WORKSPACE
    assert f(M=0, q=None) == dl.OK and f(N=0, q=None) == dl.OK
    assert dl.lora_adapters_workspace_bytes(-1, 4) == 0 and dl.lora_adapters_workspace_bytes(1, 257) == 0


@pytest.mark.parametrize("i4", [False, True])
def test_adapters_more_threads_than_a_launch_has(dl, i4):
    # 2^19 windows of 64 rows by 16 tiles of ranks: 2^23 workgroups of 512 threads
    assert _adapt(dl, M=1 << 25, r=256, N=1, wsb=1 << 62, i4=i4) == dl.ERR_SHAPE and "launch" in dl.last_error()
    # 2^15 windows by 2^9 blocks of columns: 2^24 workgroups of 256
    assert _adapt(dl, M=1 << 21, r=2, N=1 << 17, wsb=1 << 62, i4=i4) == dl.ERR_SHAPE and "launch" in dl.last_error()


def test_odd_rank_int4(dl):
    assert _adapt(dl, r=3, i4=True) == dl.ERR_SHAPE and "even" in dl.last_error()


def test_binding_refuses_host_tensors(dl):
    import torch
    z = torch.zeros
    with pytest.raises(ValueError):
        dl.ssm_prompt(z(4, 400), z(2, dtype=torch.int32), z(1, 4, 192), z(1, 1, 64, 64), z(192, 4), z(192), z(1), z(1),
                      z(1), d_state=64)
    with pytest.raises(ValueError):
        dl.ssm_step_slots(z(4, 400), z(4, dtype=torch.int32), z(4, dtype=torch.int32), z(1, 4, 192), z(1, 1, 64, 64),
                          z(192, 4), z(192), z(1), z(1), z(1), d_state=64)
    with pytest.raises(ValueError):
        dl.lora_adapters(z(1, 64, dtype=torch.int8), z(1), z(1, dtype=torch.int32), z(1, 4, 64, dtype=torch.int8),
                         z(1, 8, 4, dtype=torch.int8), z(1, 8), z(1, 8))


# ---------------------------------------------------------------- pins of the reference
def _params(rng, H, N):
    cd = 64 * H + 2 * N
    f = np.float32
    return dict(conv_w=rng.uniform(-0.5, 0.5, (cd, 4)).astype(f), conv_b=rng.uniform(-0.1, 0.1, cd).astype(f),
                dt_bias=rng.uniform(-6.9, -2.3, H).astype(f), A_log=rng.uniform(0, 2.77, H).astype(f),
                D=rng.uniform(0.5, 1.5, H).astype(f))


def test_reference_is_the_steps():
    """The reference token by token against the library's C oracle of a step."""
    import dfssm_synth as S
    import oracle
    oracle.build()
    o = oracle.get()
    M, d_model, N, L = 1, 64, 64, 6
    p = S.mamba_params(d_model, N, 64, key=(900,))
    st = S.mamba_state(M, d_model, N, 64, key=(900,))
    dm = S.mamba_dims(d_model, N, 64)
    rng = np.random.default_rng(5)
    zx = rng.standard_normal((L, 2 * dm["d_inner"] + 2 * N + dm["nheads"])).astype(np.float32)
    conv, ssm = st["conv_state"].copy(), st["ssm_state"].copy()
    pos = 9
    ring = np.zeros((4, conv.shape[1]))
    for j in range(4):
        ring[(pos - 4 + j) & 3] = conv[0, :, j]
    ref = R.scan(zx, p, ring, ssm[0], pos, N)
    for t in range(L):
        y, _, conv, ssm = o.ssm_step(zx[t:t + 1], conv, ssm, p["conv_w"], p["conv_b"], p["dt_bias"], p["A_log"],
                                     p["D"], dm["d_inner"], N, 64)
        assert np.all(np.abs(y[0] - ref["y"][t]) <= ref["y_err"][t])
    assert np.all(np.abs(ssm[0] - ref["state"]) <= ref["state_err"])
    for j in range(4):
        assert np.array_equal(ref["ring"][(pos + L - 4 + j) & 3], conv[0, :, j])


def test_bound_is_above_fp32_and_below_mistakes():
    """An fp32 evaluation of the recurrence stays inside the bound; dropping one
    tap, one token of the decay or the skip leaves it."""
    rng = np.random.default_rng(6)
    H, N, L = 2, 64, 70
    p = _params(rng, H, N)
    zx = rng.standard_normal((L, 2 * 64 * H + 2 * N + H)).astype(np.float32)
    ref = R.scan(zx, p, np.zeros((4, 64 * H + 2 * N)), np.zeros((H, 64, N)), 0, N)

    def fp32(skip=1.0, tap=1.0, late=0):
        f = np.float32
        di, cd = 64 * H, 64 * H + 2 * N
        u = np.concatenate([np.zeros((3, cd), f), zx[:, di:di + cd]])
        w = p["conv_w"].copy()
        w[:, 0] *= f(tap)
        v = p["conv_b"] + sum(w[:, j] * u[j:j + L] for j in range(4))
        s = (v / (f(1) + np.exp(-v))).astype(f)
        dt = np.log1p(np.exp(zx[:, di + cd:] + p["dt_bias"])).astype(f)
        dA = np.exp(dt * -np.exp(p["A_log"])).astype(f)
        h, out = np.zeros((H, 64, N), f), np.zeros((L, di), f)
        for t in range(L):
            x = s[t, :di].reshape(H, 64)
            h = h * dA[max(t - late, 0)][:, None, None] + (dt[t][:, None] * x)[:, :, None] * s[t, di:di + N]
            out[t] = ((h * s[t, di + N:]).sum(-1) + f(skip) * p["D"][:, None] * x).reshape(-1)
        return out
    R.assert_close(fp32(), ref["y"], ref["y_err"], ref["y_rms"], "fp32")
    for wrong in (dict(skip=0.999), dict(tap=0.0), dict(late=1)):
        with pytest.raises(AssertionError):
            R.assert_close(fp32(**wrong), ref["y"], ref["y_err"], ref["y_rms"], "wrong")


def test_halves_cost_ordinary_inputs_nothing():
    """Where no value is far above the others of its 64 tokens, what the halves of
    the prompts' products lose under a shared exponent is lost in scan's bounds."""
    rng = np.random.default_rng(7)
    for H, N, L, pos in ((2, 64, 200, 5), (1, 128, 65, 0), (2, 128, 1, 3)):
        p = _params(rng, H, N)
        zx = rng.standard_normal((L, 2 * 64 * H + 2 * N + H)).astype(np.float32)
        ring, state = rng.standard_normal((4, 64 * H + 2 * N)), 0.5 * rng.standard_normal((H, 64, N))
        ref, (y, h) = R.scan(zx, p, ring, state, pos, N), R.wide(zx, p, ring, state, pos, N)
        assert y.mean() <= 1e-4 * ref["y_err"].mean() and h.mean() <= 1e-4 * ref["state_err"].mean()
