"""AdamW groups (parameters outside the low-rank path) against the plain numpy forms."""
import ctypes as C
import subprocess

import numpy as np
import pytest
import torch

from paper_2602_04396_b200 import adamw, lordo
from paper_2602_04396_b200 import build as lbuild
from tests import tables_reference as ref

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative
# A worker's gradient norm is a sum of squares: a thread adds eight of them one after another in fp32 (relative 8 half steps of the sum, 64 of
# them would be covered too), the rest is fp64; its root halves that, and the coefficient adds a rounding.
COEF = 40 * 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    lbuild.build()
    return lordo.load_library()


# ---------------------------------------------------------------------------------------------
# no GPU
# ---------------------------------------------------------------------------------------------
def test_reference_is_adamw():
    """The plain step with omega = 1 against torch.optim.AdamW in fp64, from zero moments."""
    rng = np.random.default_rng(0)
    w = torch.from_numpy(rng.standard_normal(50)).requires_grad_()
    opt = torch.optim.AdamW([w], lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    W, m, v = w.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for s in range(1, 6):
        g = rng.standard_normal(50)
        w.grad = torch.from_numpy(g)
        opt.step()
        W, m, v, _ = ref.adamw(W, m, v, g, 0.01, 0.9, 0.99, 1.0, 1e-6, 0.1, s)
    assert np.allclose(W, w.detach().numpy(), rtol=0, atol=1e-14)


def test_reference_codes():
    """Codes are E4M3 numbers, a block's largest lies in [128, 256] of its scale, the mean over all 16-bit draws is the value itself."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal(600) * np.exp2(rng.integers(-30, 5, 600).astype(float))
    x[256:512] = 0.0
    q, e, _ = ref.round8(x, rng.integers(0, 65536, 600), False)
    assert np.array_equal(torch.from_numpy(q).float().to(torch.float8_e4m3fn).double().numpy(), q)
    assert e[1] == -126 and not q[256:512].any()
    for b in (0, 2):
        assert 128 <= np.abs(q[256 * b:256 * b + 256]).max() <= 256
    u = np.arange(65536)
    one = np.zeros(256)
    one[0] = 200.0
    for value in (0.77, 3.3e-3, 177.3, 1.0):
        got = [ref.round8(np.concatenate([[value], one[:255]]), np.concatenate([[int(k)], np.zeros(255, int)]), False)[0][0] for k in u[::257]]
        step = ref.grid(np.array([value]))[0]
        assert abs(np.mean(got) - value) <= step / 128


def test_configurations_are_checked(lib):
    def query(tensors=((100, 0, 0, 0.0),), **kw):
        arr = (lordo._Tensor * len(tensors))(*[lordo._Tensor(*t) for t in tensors])
        base = dict(n_tensors=len(tensors), tensors=arr, K=2, w_dtype=0, g_dtype=1, states=1, beta2=0.999, eps=1e-8, clip_rho=1.0, clip_scope=0, sync=1,
                    sync_m=1, sync_v=1, outer=1, outer_lr=0.7, outer_momentum=0.9, seed=1)
        base.update(kw)
        out = C.c_size_t(0)
        rc = lib.lordo_adamw_query_workspace(C.byref(lordo._AdamWConfig(*[base[f[0]] for f in lordo._AdamWConfig._fields_])), C.byref(out))
        return rc or out.value

    plain = query()
    assert plain > 8
    assert query(K=0) == 1 and query(K=65) == 1 and query(w_dtype=2) == 1 and query(g_dtype=-1) == 1 and query(states=2) == 1
    assert query(beta2=1.0) == 1 and query(eps=0.0) == 1 and query(eps=float("nan")) == 1 and query(clip_scope=2) == 1 and query(outer=2) == 1
    assert query(n_tensors=0) == 1
    assert query(((0, 0, 0, 0.0),)) == 2 and query(((100, 7, 5, 0.0),)) == 2 and query(((100, 0, 5, 0.0),)) == 2
    assert query(((100, 0, 0, float("inf")),)) == 1
    assert query(((2 ** 41, 0, 0, 0.0),)) == 8 and query(((2 ** 40, 0, 0, 0.0),) * 8, K=64) == 8
    # a table's scratch: the sums of up to 50 rows of 10 for both workers
    assert query(((100, 10, 50, 0.0),)) >= plain + 4 * 2 * 50 * 10
    assert lib.lordo_adamw_query_workspace(None, None) == 1


def test_division_by_multiplication(tmp_path):
    """The rule by which a step finds the row of an element (csrc/lordo_plan.h): at multiples of the divisor, beside them and at the ends."""
    src, so = str(tmp_path / "d.cpp"), str(tmp_path / "d.so")
    with open(src, "w") as f:
        f.write('#include "lordo_plan.h"\nextern "C" unsigned quotient(unsigned x, unsigned q) {\n  const lordo::Divider d = lordo::divider(q);\n'
                '  return (unsigned)(((unsigned long long)x * d.mul) >> (31 + d.shift));\n}\n')
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", lbuild.CSRC, "-o", so, src], check=True)
    f = C.CDLL(so).quotient
    f.restype, f.argtypes = C.c_uint, [C.c_uint, C.c_uint]
    rng = np.random.default_rng(0)
    for q in [1, 2, 3, 5, 7, 96, 125, 256, 1000, 2 ** 20 - 1, 2 ** 20, 2 ** 20 + 1, 2 ** 21 - 1, 2 ** 24 - 1, 2 ** 24] + rng.integers(1, 2 ** 21, 200).tolist():
        k = rng.integers(0, (2 ** 31 - 2) // q + 1, 40)
        for x in [0, q - 1, q, 2 ** 31 - 1, 2 ** 31 - 2] + (k * q).tolist() + np.maximum(k * q - 1, 0).tolist():
            assert f(x, q) == x // q, (x, q)


def test_null_arguments_are_rejected(lib):
    assert lib.lordo_adamw_init(None, None, None, 0, None, None) == 1
    assert lib.lordo_adamw_step(None, None, 0.1, 0.9, 1.0, None, None) == 1
    assert lib.lordo_adamw_outer_step(None, None) == 1
    assert lib.lordo_adamw_destroy(None) == 1
    assert lib.lordo_adamw_launch_count(None) == -1
    assert lib.lordo_adamw_get_counters(None, None) == 1 and lib.lordo_adamw_set_counters(None, None) == 1


def test_binding_refuses_bad_groups():
    with pytest.raises(ValueError):
        adamw.AdamW([], 1)
    with pytest.raises(ValueError):
        adamw.AdamW([torch.zeros(3)], 1, states="4bit")
    with pytest.raises(ValueError):
        adamw.AdamW([torch.zeros(3), torch.zeros(3, dtype=torch.bfloat16)], 1)


# ---------------------------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------------------------
SETS = {
    "one": [(1,)],
    "tiny": [(3,), (1,), (7,), (8,), (9,)],
    "odd": [(1003, 3), (257,), (256,), (255,), (4097,)],
    "pieces": [(8192,), (8193,), (40000,), (70001,)],
    "many": [(24,)] * 600,
}


def group(shapes, K, draw, w="f32", **kw):
    gen = torch.Generator().manual_seed(draw)
    W0 = [torch.randn(s, generator=gen).mul_(0.5).to(DT[w]) for s in shapes]
    return adamw.AdamW(W0, K, weight_decay=[0.1 * (i % 2) for i in range(len(shapes))], **kw)


def gradients(shapes, K, seed, dt, std=0.3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((K,) + s, device="cuda", generator=gen).mul_(std).to(DT[dt]) for s in shapes]


def check_moments8(codes, scales, want, err, u, positive):
    """[K] codes against the rounding of fp64 values that are known to `err`: the same but where that could move the argument over a border,
    and then by one step. A scale may differ where the block's largest is that near to a power of two."""
    for k in range(len(want)):
        c, e = ref.to64(codes[k]).reshape(-1), np.log2(ref.to64(scales[k]))
        x, d = want[k].reshape(-1), err[k].reshape(-1)
        blocks = lambda a: np.pad(a, (0, -a.size % 256)).reshape(-1, 256)
        q, e_ref, border = ref.round8(x, u[k], positive)
        top = np.maximum(blocks(np.abs(x)).max(axis=1), 1e-300)
        edge = np.abs(top - np.exp2(np.rint(np.log2(top)))) <= blocks(d).max(axis=1)
        assert np.array_equal(e[~edge], e_ref[~edge])
        unit = np.exp2(e_ref.repeat(256)[:x.size].astype(float))
        step = ref.grid(np.abs(x) / unit)
        differ = np.repeat(e == e_ref, 256)[:x.size] & (c != q)
        assert (np.abs(c - q)[differ] <= 2 * step[differ]).all()
        assert (border[differ] <= (d / unit / step)[differ] + 2.0 ** -18).all()


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("w,g", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("K,rho,scope,omega", [(1, 0.0, 0, 1.0), (3, 2.0, 0, 0.9), (2, 0.7, 1, 1.0)])
def test_steps(name, w, g, states, K, rho, scope, omega):
    """Three steps, each compared with the plain step from the state that the kernel itself had before it. m and v are sums of two products:
    four roundings, and the coefficient's. The update's quotient: those of m and v, half of v's under the root, five more."""
    shapes = SETS[name]
    opt = group(shapes, K, 1, w, g_dtype=DT[g], states=states, beta2=0.99, eps=1e-3, clip_rho=rho, clip_scope=scope, seed=77)
    lr, b1, b2, eps = 0.01, 0.9, 0.99, 1e-3
    om = omega
    for s in range(1, 4):
        G = gradients(shapes, K, 10 + s, g)
        G64 = [ref.to64(x).reshape(K, -1) for x in G]
        coef = ref.clip(G64, rho, scope)
        W0 = [ref.to64(x).reshape(K, -1) for x in opt.W]
        m0, v0 = ([ref.to64(x).reshape(K, -1) for x in y] for y in (opt.m, opt.v))
        if states == "8bit":
            wide = lambda c, sc: c * np.repeat(ref.to64(sc), 256, axis=1)[:, :c.shape[1]]
            m0 = [wide(x, sc) for x, sc in zip(m0, opt.ms)]
            v0 = [wide(x, sc) ** 2 for x, sc in zip(v0, opt.vs)]
        opt.step(G, 0.01, 0.9, omega)
        if rho > 0:
            assert (np.abs(ref.to64(opt.clip_coefficients()) - coef) <= COEF * coef).all()
        for i in range(len(shapes)):
            wd = ref.f32(0.1 * (i % 2))
            gr = G64[i] * coef[i][:, None]
            W, m, v, up = ref.adamw(W0[i], m0[i], v0[i], gr, lr, b1, b2, om, eps, wd, s)
            dm = 4 * HALF["f32"] * (np.abs(b1 * m0[i]) + np.abs((1 - b1) * gr)) + COEF * np.abs((1 - b1) * gr)
            dv = (6 * HALF["f32"] + 2 * COEF) * v
            if states == "f32":
                assert (np.abs(ref.to64(opt.m[i]).reshape(K, -1) - m) <= dm).all()
                assert (np.abs(ref.to64(opt.v[i]).reshape(K, -1) - v) <= dv).all()
            else:
                u = [ref.random16(77, 3, s, i * K + k, W.shape[1]) for k in range(K)]
                check_moments8(opt.m[i], opt.ms[i], m, dm + 4 * HALF["f32"] * np.abs(m), u, False)
                check_moments8(opt.v[i], opt.vs[i], np.sqrt(v), (8 * HALF["f32"] + COEF) * np.sqrt(v), [ref.second16(x) for x in u], True)
            D = np.sqrt(v / (1 - b2 ** s)) + eps
            dup = om / (1 - b1 ** s) * dm / D + ((1 - om) * np.abs(gr) / D) * COEF + np.abs(up) * (12 * HALF["f32"] + COEF)
            dup += 4 * HALF["f32"] * (np.abs(om * m / (1 - b1 ** s)) + np.abs((1 - om) * gr)) / D
            off = lr * (dup + 4 * HALF["f32"] * np.abs(up)) + 4 * HALF["f32"] * np.abs(W0[i])
            got = ref.to64(opt.W[i]).reshape(K, -1)
            assert (np.abs(got - W) <= off + HALF[w] * (np.abs(W) + off)).all(), (i, np.abs(got - W).max())
    assert opt.poll_status() == 0 and opt.counters() == [3, 0]
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("std", [1e-14, 1e-6, 30.0, 1e6])
@pytest.mark.parametrize("kind", ["spread", "half empty", "one"])
def test_magnitudes_in_8_bits(std, kind):
    """Two steps on gradients from far below to far above 1: blocks whose magnitudes lie 30 powers of two apart, blocks with rows that never had a
    gradient beside others, blocks with one element that had. Checked as the other steps are.

    v is formed in fp32 and counts as 0 below 2^-126, the smallest normal number: gradients of 1e-14 * 2^-30 have squares of 1e-46, which fp32 does
    not hold. Its operands may be subnormal, each off by 2^-150: of a v at 2^-126 that is 2^-23, so v within 1e-6 of that border may go either way."""
    K, n = 2, 256 * 40 + 24
    least = 2.0 ** -126
    gen = torch.Generator(device="cuda").manual_seed(3)
    opt = adamw.AdamW([torch.ones(n)], K, states="8bit", beta2=0.99, eps=std * 1e-3, seed=21)
    W0 = ref.to64(opt.W[0])
    m0 = v0 = np.zeros((K, n))
    for s in range(1, 3):
        g = torch.randn(K, n, device="cuda", generator=gen) * std
        if kind == "spread":
            g *= torch.exp2(-30.0 * torch.rand(K, n, device="cuda", generator=gen))
        elif kind == "half empty":
            g[:, (torch.arange(n, device="cuda") // 100) % 2 == 0] = 0.0
        else:
            g[:, torch.arange(n, device="cuda") % 300 != 7] = 0.0
        opt.step([g], 0.01, 0.9)
        G = ref.to64(g)
        raw = 0.99 * v0 + 0.01 * G * G
        assert not (np.abs(raw / least - 1) < 1e-6).any()  # none at the border among these
        W, m, v, up = ref.adamw(W0, m0, v0, G, 0.01, 0.9, 0.99, 1.0, std * 1e-3, 0.0, s, least=least)
        dm = 4 * HALF["f32"] * (np.abs(0.9 * m0) + np.abs(0.1 * G))
        u = [ref.random16(21, 3, s, k, n) for k in range(K)]
        check_moments8(opt.m[0], opt.ms[0], m, dm + 4 * HALF["f32"] * np.abs(m), u, False)
        check_moments8(opt.v[0], opt.vs[0], np.sqrt(v), 8 * HALF["f32"] * np.sqrt(v), [ref.second16(x) for x in u], True)
        got = ref.to64(opt.W[0])
        D = np.sqrt(v / (1 - 0.99 ** s)) + std * 1e-3
        off = 0.01 * (dm / (1 - 0.9 ** s) / D + 16 * HALF["f32"] * np.abs(up)) + 2 * HALF["f32"] * np.abs(W)
        assert (np.abs(got - W) <= off).all()
        assert torch.equal(opt.v[0].float() != 0, torch.from_numpy(v != 0).cuda())  # what had a gradient never comes to 0, the rest is
        wide = lambda c, sc: ref.to64(c) * np.repeat(ref.to64(sc), 256, axis=1)[:, :n]
        W0, m0, v0 = got, wide(opt.m[0], opt.ms[0]), wide(opt.v[0], opt.vs[0]) ** 2
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_two_tables_by_tokens_and_many_workers(states):
    """Token and position tables in one step, fewer tokens than declared, 64 workers; then the same step with dense gradients for one of them:
    coefficients as for the dense gradients (test_norm_of_a_gradient_by_tokens derives their bound), the rest from outside."""
    from paper_2602_04396_b200 import embedding
    K = 64
    shapes = [(40, 24), (33,), (16, 24)]
    a = group(shapes, K, 1, states=states, tables={0: 50, 2: 16}, clip_rho=0.5, seed=4)
    b = group(shapes, K, 1, states=states, clip_rho=0.5, seed=4)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for s in range(2):
        tok = torch.randint(0, 40, (K, 2, 8), device="cuda", generator=gen)
        pos = torch.arange(16, device="cuda").view(1, 2, 8).expand(K, 2, 8).contiguous()
        dY = torch.randn(K, 2, 8, 24, device="cuda", generator=gen)
        g1 = gradients([(33,)], K, s, "f32")[0]
        dense = [embedding.embedding_grad(dY, x, n, K=K) for x, n in ((tok, 40), (pos, 16))]
        a.step([adamw.TokenGrad(tok, dY), g1, adamw.TokenGrad(pos, dY)], 0.01)
        b.step([dense[0], g1, dense[1]], 0.01)
        ca, cb = ref.to64(a.clip_coefficients()), ref.to64(b.clip_coefficients())
        assert (np.abs(ca - cb) <= (2 * COEF + 40 * 2.0 ** -24) * cb).all()
        coef = torch.rand(K, device="cuda", generator=gen)
        a.step([adamw.TokenGrad(tok, dY), g1, dense[1]], 0.01, coef=coef)
        b.step([dense[0], g1, dense[1]], 0.01, coef=coef)
    c = group(shapes, K, 1, states=states, tables={0: 50, 2: 16}, seed=4)
    d = group(shapes, K, 1, states=states, seed=4)
    c.step([adamw.TokenGrad(tok, dY), g1, adamw.TokenGrad(pos, dY)], 0.01)
    d.step([dense[0], g1, dense[1]], 0.01)
    for x in c.storage:
        assert torch.equal(c.storage[x].view(torch.uint8), d.storage[x].view(torch.uint8)), x


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_elements_behind_two_to_the_32nd(states):
    """Two workers of 2^31 + 24 elements each (and a small tensor behind them): the last ones move as those of a small group with the same
    gradients, bit for bit where rounding does not look at the element's number, and the synchronisation reaches them."""
    n, tail = 2 ** 31 + 24, 24
    K = 2
    big = adamw.AdamW([torch.zeros(n, dtype=torch.bfloat16), torch.zeros(9, dtype=torch.bfloat16)], K, states=states, outer=lordo.OUTER_AVG)
    small = adamw.AdamW([torch.zeros(tail, dtype=torch.bfloat16), torch.zeros(9, dtype=torch.bfloat16)], K, states=states, outer=lordo.OUTER_AVG)
    G = [torch.zeros(K, n, device="cuda", dtype=torch.bfloat16), torch.ones(K, 9, device="cuda", dtype=torch.bfloat16)]
    g = torch.randn(K, tail, device="cuda").to(torch.bfloat16)
    G[0][:, -tail:] = g
    coef = torch.ones(K, device="cuda")
    big.step(G, 0.1, coef=coef)
    small.step([g, G[1]], 0.1, coef=coef)
    assert torch.equal(big.W[0][:, -tail:], small.W[0]) and torch.equal(big.W[1], small.W[1])
    assert not big.W[0][:, n // 2:n // 2 + 1000].any() and not big.W[0][:, :1000].any()
    if states == "f32":
        assert torch.equal(big.m[0][:, -tail:], small.m[0]) and torch.equal(big.v[0][:, -tail:], small.v[0])
    else:  # one block of 24 elements in either
        assert torch.equal(big.ms[0][:, -1].float(), small.ms[0][:, -1].float())
        assert (big.v[0][:, -tail:].float() > 0).all() and not big.v[0][:, -tail - 1000:-tail].view(torch.uint8).any()
    big.outer_step()
    small.outer_step()
    assert torch.equal(big.W[0][:, -tail:], small.W[0])
    big.close(), small.close()


@pytest.mark.gpu
@pytest.mark.parametrize("V,d,T", [(50, 8, 1), (300, 40, 700), (97, 33, 64), (5, 16, 3000), (3000, 264, 33), (700, 128, 0)])
@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gradient_by_tokens(V, d, T, states, dt):
    """A table's gradient by its tokens against the same sums handed over as a dense fp32 gradient: the moments and weights are those of a
    group whose gradients are in fp32, bit for bit (the sums are the same kernel's), but for the norm, whose order differs. So clipping is
    off here, and coefficients come from outside."""
    K = 2
    shapes = [(9,), (V, d), (3, 5)]
    kw = dict(states=states, beta2=0.99, eps=1e-4, seed=3)
    a = group(shapes, K, 2, dt, g_dtype=DT[dt], tables={1: T + 3}, **kw)
    b = group(shapes, K, 2, dt, g_dtype=torch.float32, **kw)
    coef = torch.tensor([0.5, 0.25], device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(V)
    from paper_2602_04396_b200 import embedding
    for s in range(2):
        tokens = torch.randint(-1, V + 1, (K, T), device="cuda", generator=gen, dtype=torch.int64 if s else torch.int32)
        dY = torch.randn(K, T, d, device="cuda", generator=gen).to(DT[dt])
        G = gradients(shapes, K, s, dt)
        dense = embedding.embedding_grad(dY, tokens, V, scale=1.7, K=K, out_dtype=torch.float32)
        a.step([G[0], adamw.TokenGrad(tokens, dY, 1.7), G[2]], 0.01, 0.9, coef=coef)
        b.step([G[0].float(), dense, G[2].float()], 0.01, 0.9, coef=coef)
        for x in a.storage:
            assert torch.equal(a.storage[x].view(torch.uint8), b.storage[x].view(torch.uint8)), x
    a.step(G, 0.01)  # a dense gradient for the same table
    b.step([x.float() for x in G], 0.01)
    assert torch.equal(a.storage["W"], b.storage["W"])
    a.close(), b.close()


@pytest.mark.gpu
@pytest.mark.parametrize("V,d,T", [(50, 8, 1), (300, 40, 700), (97, 33, 64), (5, 16, 3000), (700, 128, 0)])
@pytest.mark.parametrize("scope", [0, 1])
def test_norm_of_a_gradient_by_tokens(V, d, T, scope):
    """Its share of the clip norm. Every sum of L terms is off by L half steps of its magnitudes; here that is bounded over the table by
    the largest count."""
    K = 3
    shapes = [(V, d), (1000,)]
    opt = group(shapes, K, 2, g_dtype=torch.bfloat16, tables={0: T}, clip_rho=0.8, clip_scope=scope)
    rng = np.random.default_rng(V)
    tok = rng.integers(-1, V, (K, T))
    dY = torch.randn(K, T, d, device="cuda").to(torch.bfloat16)
    G = gradients(shapes, K, 5, "bf16", std=0.05)
    opt.step([adamw.TokenGrad(torch.from_numpy(tok).cuda(), dY, 0.5), G[1]], 0.01)
    y = ref.to64(dY)
    want = ref.clip([ref.table_grad(tok, y, V, 0.5).reshape(K, -1), ref.to64(G[1])], 0.8, scope)
    size = np.sqrt((ref.table_grad(tok, np.abs(y), V, 0.5) ** 2).sum(axis=(1, 2)))
    norm = np.sqrt((ref.table_grad(tok, y, V, 0.5) ** 2).sum(axis=(1, 2)))
    terms = max([np.bincount(t[t >= 0], minlength=1).max() for t in tok] + [1])
    off = COEF + (terms + 2) * 2.0 ** -24 * (size / np.maximum(norm, 1e-30)).max()
    assert (np.abs(ref.to64(opt.clip_coefficients()) - want) <= off * want).all()
    assert opt.poll_status() == 0
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["one", "tiny", "odd", "many"])
@pytest.mark.parametrize("w", ["f32", "bf16"])
@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("K,outer,sync", [(1, 0, (True, True)), (4, 1, (True, False)), (5, 1, (True, True)), (3, 0, (False, True))])
def test_outer_step(name, w, states, K, outer, sync):
    """A step that drives the workers apart, then the synchronisation, twice. Means of K values: K roundings; the outer update a few more."""
    shapes = SETS[name]
    opt = group(shapes, K, 4, w, states=states, eps=1e-3, outer=outer, outer_lr=0.7, outer_momentum=0.9, sync_m=sync[0], sync_v=sync[1], seed=9)
    eta, mu = 0.7, 0.9
    for r in range(2):
        opt.step(gradients(shapes, K, 20 + r, w), 0.05)
        before = {x: [ref.to64(t) for t in getattr(opt, x)] for x in ("W", "m", "v", "ms", "vs", "X0", "B")}
        opt.outer_step()
        for i in range(len(shapes)):
            W = before["W"][i].reshape(K, -1)
            x0, B = before["X0"][i].reshape(-1), before["B"][i].reshape(-1)
            delta = x0 - W.mean(axis=0)
            e = HALF["f32"] * ((K + 1) * np.abs(W).mean(axis=0) + 2 * np.abs(x0))
            if outer == lordo.OUTER_NESTEROV:
                B = mu * B + delta
                eb = e + 4 * HALF["f32"] * (np.abs(B) + np.abs(delta) + np.abs(before["B"][i].reshape(-1)))
                assert (np.abs(ref.to64(opt.B[i]).reshape(-1) - B) <= eb).all()
                x1 = x0 - eta * (delta + mu * B)
                ex = e + eb + 6 * HALF["f32"] * (np.abs(x0) + np.abs(delta) + np.abs(B))
            else:
                x1 = x0 - delta
                ex = e + 2 * HALF["f32"] * (np.abs(x0) + np.abs(delta))
            assert (np.abs(ref.to64(opt.X0[i]).reshape(-1) - x1) <= ex).all()
            for k in range(K):
                assert torch.equal(opt.W[i][k], opt.X0[i].to(DT[w]))
            for x, on, second in (("m", sync[0], False), ("v", sync[1], True)):
                now = getattr(opt, x)[i]
                old = before[x][i].reshape(K, -1)
                if not on:
                    assert np.array_equal(ref.to64(now).reshape(K, -1), old)
                    continue
                if states == "f32":
                    mean = old.mean(axis=0)
                    assert (np.abs(ref.to64(now).reshape(K, -1) - mean) <= (K + 1) * HALF["f32"] * np.abs(old).mean(axis=0)).all()
                    continue
                old = old * np.repeat(before[x + "s"][i], 256, axis=1)[:, :old.shape[1]]
                mean = np.sqrt((old ** 2).mean(axis=0)) if second else old.mean(axis=0)
                u = ref.random16(9, 4, r, i, old.shape[1])
                err = (K + 4) * HALF["f32"] * (mean if second else np.abs(old).mean(axis=0))  # of a mean of K values, its square and root
                for k in range(K):
                    check_moments8(now[k:k + 1], getattr(opt, x + "s")[i][k:k + 1], [mean], [err], [ref.second16(u) if second else u], second)
                    assert torch.equal(now[k].view(torch.uint8), now[0].view(torch.uint8))
    assert opt.counters() == [2, 2]
    opt.close()


@pytest.mark.gpu
def test_slow_averages_move_in_8_bits():
    """beta2 = 0.999 and a gradient that vanishes: v falls by 0.1 % a step, a fortieth of the smallest distance of codes of its root. After
    700 steps the mean of sqrt(v) over 65536 elements is sqrt(0.999^700) = 0.7045 of the start's: within 2 % (a walk of 65536 elements of at most
    12.5 % a step with probability 0.4 %: 0.25 per element after 700 steps, 0.001 for their mean, and as much for its curvature)."""
    n = 65536
    opt = adamw.AdamW([torch.zeros(n)], 1, states="8bit", seed=5)
    opt.step([torch.full((1, n), 0.37, device="cuda")], 0.0)
    start = float((opt.v[0].float() * opt.vs[0].float().repeat_interleave(256, dim=1)).mean())
    none = torch.zeros(1, n, device="cuda")
    for _ in range(700):
        opt.step([none], 0.0)
    end = float((opt.v[0].float() * opt.vs[0].float().repeat_interleave(256, dim=1)).mean())
    assert abs(end / start / 0.999 ** 350 - 1) < 0.02, (end / start, 0.999 ** 350)
    assert opt.m[0].float().abs().max() * float(opt.ms[0].float().max()) < 1e-20  # beta1 = 0.9
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_nonfinite_gradients(states):
    """One worker's infinity sets the flag, becomes NaN in that element's own worker and stays away from the others."""
    opt = group([(300,), (77,)], 2, 1, states=states, clip_rho=1.0)
    G = gradients([(300,), (77,)], 2, 1, "f32")
    G[0][1, 5] = float("inf")
    opt.step(G, 0.01)
    assert opt.poll_status() == lordo.FLAG_NONFINITE_GRAD
    assert torch.isnan(opt.W[0][1, 5]) and torch.isfinite(opt.W[0][0]).all() and torch.isfinite(opt.W[1]).all()
    assert torch.isnan(opt.m[0][1, 5].float()) and torch.isnan(opt.v[0][1, 5].float())
    opt.clear_status()
    assert opt.poll_status() == 0
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_checkpoint_and_repetition(states):
    """Two runs of the same schedule give the same bits, and so does one that is restored half way from the storage and the counters."""
    shapes = [(40, 24), (300,), (7,)]
    kw = dict(states=states, clip_rho=1.0, outer=lordo.OUTER_NESTEROV, outer_lr=0.7, outer_momentum=0.9, seed=8, tables={0: 30})

    def go(opt, first, last):
        for s in range(first, last):
            gen = torch.Generator(device="cuda").manual_seed(s)
            tok = torch.randint(0, 40, (2, 30), device="cuda", generator=gen)
            G = gradients(shapes, 2, s, "f32")
            opt.step([adamw.TokenGrad(tok, torch.randn(2, 30, 24, device="cuda", generator=gen))] + G[1:], 0.01)
            if s % 2:
                opt.outer_step()

    a, b, c = (group(shapes, 2, 1, **kw) for _ in range(3))
    go(a, 0, 6)
    go(b, 0, 3)
    for x, y in b.storage.items():
        c.storage[x].view(torch.uint8).copy_(y.view(torch.uint8))
    c.set_counters(b.counters())
    go(b, 3, 6)
    go(c, 3, 6)
    for x in a.storage:
        assert torch.equal(a.storage[x].view(torch.uint8), b.storage[x].view(torch.uint8)), x
        assert torch.equal(a.storage[x].view(torch.uint8), c.storage[x].view(torch.uint8)), x
    assert a.counters() == [6, 3]


@pytest.mark.gpu
def test_streams():
    """Steps on a stream of their own, two groups at once: the same bits as one after the other."""
    shapes = [(5000,), (300, 16)]
    ref_opts = [group(shapes, 2, i, clip_rho=1.0, states=s, tables={1: 64}) for i, s in ((1, "f32"), (2, "8bit"))]
    opts = [group(shapes, 2, i, clip_rho=1.0, states=s, tables={1: 64}) for i, s in ((1, "f32"), (2, "8bit"))]
    tok = torch.randint(0, 300, (2, 64), device="cuda")
    G = [gradients(shapes, 2, 9, "f32")[0], adamw.TokenGrad(tok, torch.randn(2, 64, 16, device="cuda"))]
    streams = [torch.cuda.Stream() for _ in opts]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for o in ref_opts:
            o.step(G, 0.01)
        for o, s in zip(opts, streams):
            o.step(G, 0.01, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(ref_opts, opts):
        for x in a.storage:
            assert torch.equal(a.storage[x].view(torch.uint8), b.storage[x].view(torch.uint8)), x


@pytest.mark.gpu
def test_refusals():
    opt = group([(20, 8), (5,)], 2, 1, g_dtype=torch.bfloat16, tables={0: 4})
    G = gradients([(20, 8), (5,)], 2, 1, "bf16")
    tok, dY = torch.zeros(2, 4, device="cuda", dtype=torch.int64), torch.zeros(2, 4, 8, device="cuda", dtype=torch.bfloat16)
    bad = [lambda: opt.step(G[:1], 0.1), lambda: opt.step([G[0].float(), G[1]], 0.1), lambda: opt.step([G[0][:1], G[1]], 0.1),
           lambda: opt.step([G[0].cpu(), G[1]], 0.1), lambda: opt.step([G[0].transpose(1, 2).contiguous().transpose(1, 2), G[1]], 0.1),
           lambda: opt.step([G[0], adamw.TokenGrad(tok, dY)], 0.1), lambda: opt.step([adamw.TokenGrad(tok, dY.float()), G[1]], 0.1),
           lambda: opt.step([adamw.TokenGrad(tok[:1], dY), G[1]], 0.1), lambda: opt.step([adamw.TokenGrad(tok.to(torch.int16), dY), G[1]], 0.1),
           lambda: opt.step(G, 0.1, coef=torch.ones(3, device="cuda")), lambda: opt.step(G, 0.1, coef=torch.ones(2))]
    before = opt.storage["W"].clone()
    for call in bad:
        with pytest.raises(ValueError):
            call()
    many = torch.zeros(2, 5, device="cuda", dtype=torch.int64)
    for call, code in [(lambda: opt.step([adamw.TokenGrad(many, torch.zeros(2, 5, 8, device="cuda", dtype=torch.bfloat16)), G[1]], 0.1), 1),
                       (lambda: opt.step(G, 0.1, beta1=1.0), 1), (lambda: opt.step(G, 0.1, omega=1.5), 1), (opt.outer_step, 4),
                       (lambda: opt.set_counters([-1, 0]), 1)]:
        with pytest.raises(lordo.LordoError) as e:
            call()
        assert e.value.status == code
    flat = torch.zeros(2 * 20 * 8 + 1, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(lordo.LordoError) as e:
        opt.step([flat[1:].view(2, 20, 8), G[1]], 0.1)
    assert e.value.status == 3
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        keep = before + 1
        with pytest.raises(lordo.LordoError) as e:
            opt.step(G, 0.1)
        assert e.value.status == 8
    assert torch.equal(opt.storage["W"], before) and opt.counters() == [0, 0]
    opt.step(G, 0.1)
    assert opt.poll_status() == 0
    out, names = C.c_void_p(None), ("W", "m", "v", "ms", "vs", "X0", "B")
    bufs = lordo._AdamWBuffers(*[C.cast(opt._pointers[x], C.POINTER(C.c_void_p)) if x in opt._pointers else None for x in names])
    init = lambda ws, size: opt.lib.lordo_adamw_init(C.byref(opt.cfg), C.byref(bufs), ws, size, None, C.byref(out))
    assert init(opt.workspace.data_ptr(), 16) == 5 and init(opt.workspace.data_ptr() + 16, opt.workspace_bytes) == 3 and init(None, 16) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_a_round_beside_the_low_rank_path(states):
    """One model's parameters: two matrices in a Lordo, its table and gains in a group, two rounds of H steps with the matrices' own clip
    coefficients, then both synchronised. Gradients of the table come from the lookup's. Replicas agree afterwards and everything moved."""
    from paper_2602_04396_b200 import embedding
    K, H, V, d = 3, 4, 64, 32
    gen = torch.Generator(device="cuda").manual_seed(0)
    mats = [(32, 64, 8), (64, 32, 8)]
    low = lordo.Lordo(mats, K, H, [torch.randn(m, n) * 0.02 for m, n, _ in mats], clip_rho=1.0, outer=lordo.OUTER_NESTEROV, outer_lr=0.7, outer_momentum=0.9)
    rest = adamw.AdamW([torch.randn(V, d) * 0.02, torch.ones(d)], K, states=states, tables={0: 16}, outer=lordo.OUTER_NESTEROV, outer_lr=0.7,
                       outer_momentum=0.9, seed=1)
    first = rest.storage["W"].clone()
    for _ in range(2):
        for _ in range(H):
            tok = torch.randint(0, V, (K, 16), device="cuda", generator=gen)
            x = embedding.embedding(rest.W[0], tok, scale=d ** 0.5)
            dY = x * 0.1 + torch.randn(x.shape, device="cuda", generator=gen) * 0.01
            G = [torch.randn(K, m, n, device="cuda", generator=gen) for m, n, _ in mats]
            low.inner_step(G, 0.01, 0.9, 1.0, lordo.QHM_NONE)
            rest.step([adamw.TokenGrad(tok, dY, d ** 0.5), dY.sum(dim=1)], 0.01, 0.9, coef=low.clip_coefficients()[0])
        low.outer_step()
        rest.outer_step()
        low.refresh_subspace()
        for W in rest.W + low.W:
            assert all(torch.equal(W[k], W[0]) for k in range(K)) and torch.isfinite(W).all()
    assert low.poll_status() == 0 and rest.poll_status() == 0 and rest.counters() == [2 * H, 2]
    assert (rest.storage["W"] != first).float().mean() > 0.5
    low.close(), rest.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), 1e25])
@pytest.mark.parametrize("n", [300, 4096])
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_a_nonfinite_gradient_stays_in_its_elements(states, bad, n):
    """Four steps and a synchronisation after one worker's infinity or NaN, in a block with others and in a block of nothing else: all other elements,
    and all scales, have the bits of a group whose gradients are 0 there. (1e25: v is infinite, m is not, and is its block's largest, so that 8-bit
    neighbours lose theirs: they stay finite.)"""
    K, shapes = 3, [(n,), (77,)]
    hit = torch.zeros(n, dtype=torch.bool, device="cuda")
    hit[5] = True
    hit[256:512] = n > 512
    kw = dict(states=states, eps=1e-3, seed=6, outer=lordo.OUTER_NESTEROV, outer_lr=0.7, outer_momentum=0.9)
    a, b = (group(shapes, K, 1, **kw) for _ in range(2))
    coef = torch.ones(K, device="cuda")
    for s in range(4):
        G = gradients(shapes, K, s, "f32")
        G[0][:, hit] = 0.0
        b.step(G, 0.01, coef=coef)
        if s == 0:
            G[0][1, hit] = bad
        a.step(G, 0.01, coef=coef)
        if s == 2:
            a.outer_step(), b.outer_step()
        worker = slice(0, K) if s >= 2 else slice(1, 2)
        bits = lambda x: x.view(torch.uint8 if x.element_size() == 1 else torch.int32)
        for name in ("W", "m", "v", "ms", "vs"):
            for i, (x, y) in enumerate(zip(getattr(a, name), getattr(b, name))):
                rest = ~hit if name in ("W", "m", "v") and i == 0 else slice(None)
                if abs(bad) < float("inf") and i == 0 and name not in ("v", "vs"):
                    assert torch.isfinite(x.float()[:, rest]).all(), (s, name)
                else:
                    assert torch.equal(bits(x)[:, rest], bits(y)[:, rest]), (s, name, i)
        assert not torch.isfinite(a.v[0][worker].float()[:, hit]).any()
        if not abs(bad) < float("inf"):
            assert torch.isnan(a.W[0][worker][:, hit]).all()
    a.close(), b.close()


@pytest.mark.gpu
@pytest.mark.parametrize("lr,wd", [(1e-3, 0.1), (1e-5, 0.1), (1e-6, 0.1), (2e-7, 0.1), (1e-6, 0.01)])
@pytest.mark.parametrize("omega", [1.0, 0.9])
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_weight_decay_far_below_a_step_of_the_weights(states, omega, lr, wd):
    """The change of an fp32 weight is formed apart and added once: off by half a step of the new weight, and by the roundings of the change itself.
    Those, in half steps: the moments 4 and 6 (3 under the root), the constants 5 each, the products, the root (2), the quotient (2) and the
    sums 8: at most 40 of the update, and 8 (the rates, their product, its product with the weight, the sum) of the decay. Blocks that never
    had a gradient, a last block that is not whole, and workers at odd addresses."""
    K = 2
    for n in (256 * 40 + 100, 255 * 17):
        gen = torch.Generator(device="cuda").manual_seed(n)
        opt = adamw.AdamW([torch.randn(n, generator=gen, device="cuda")], K, states=states, eps=1e-3, weight_decay=wd, seed=2)
        g = torch.randn(K, n, device="cuda", generator=gen)
        g[:, 512:1024] = 0.0
        W0 = ref.to64(opt.W[0])
        opt.step([g], lr, 0.9, omega)
        W, _, _, up = ref.adamw(W0, 0.0, 0.0, ref.to64(g), lr, 0.9, 0.999, omega, 1e-3, wd, 1)
        got = ref.to64(opt.W[0])
        step = np.spacing(np.maximum(np.abs(got), np.abs(W)).astype(np.float32)).astype(np.float64)
        off = HALF["f32"] * (40 * lr * np.abs(up) + 8 * lr * wd * np.abs(W0))
        assert (np.abs(got - W) <= step / 2 + off).all(), (np.abs(got - W) / step).max()
        opt.close()


def _junk_like(tensors):
    """Takes memory of the same sizes and fills it: with what allocations of the current stream that were given back have left."""
    return [torch.full_like(t, -1 if t.dtype in (torch.int32, torch.int64) else float("nan")) for t in tensors]


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_gradients_given_back_before_their_stream_has_come_to_them(states):
    """Steps on a stream that is still busy with earlier work (a tenth of a second), gradients, tokens and coefficients allocated anew for each and
    dropped at once, their memory taken and overwritten on the current stream: the bits of steps whose gradients were kept."""
    K, shapes = 2, [(300, 512), (70000,)]
    a, b = (group(shapes, K, 1, states=states, tables={0: 64}, seed=3) for _ in range(2))

    def make(s):
        gen = torch.Generator(device="cuda").manual_seed(s)
        tok = torch.randint(0, 300, (K, 64), device="cuda", generator=gen)
        dY = torch.randn(K, 64, 512, device="cuda", generator=gen)
        return tok, dY, torch.randn(K, 70000, device="cuda", generator=gen), torch.rand(K, device="cuda", generator=gen)

    kept = [make(s) for s in range(6)]
    for tok, dY, g, coef in kept:
        b.step([adamw.TokenGrad(tok, dY), g], 0.01, coef=coef)
    side, junk = torch.cuda.Stream(), [_junk_like(kept[0])]  # its kernels are loaded by now
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    for s in range(6):
        tok, dY, g, coef = make(s)
        torch.cuda.current_stream().synchronize()
        a.step([adamw.TokenGrad(tok, dY), g], 0.01, coef=coef, stream=side)
        del tok, dY, g, coef
        junk.append(_junk_like(kept[s]))
    torch.cuda.synchronize()
    for x in a.storage:
        assert torch.equal(a.storage[x].view(torch.uint8), b.storage[x].view(torch.uint8)), x
    a.close(), b.close()


@pytest.mark.gpu
def test_gradients_are_not_held_after_the_step():
    """On the current stream the allocator's own order is enough: a step keeps nothing that its caller has dropped."""
    import weakref
    opt = group([(50, 8), (9,)], 2, 1, tables={0: 4})
    tok, dY, g = torch.zeros(2, 4, device="cuda", dtype=torch.int64), torch.ones(2, 4, 8, device="cuda"), torch.ones(2, 9, device="cuda")
    coef = torch.ones(2, device="cuda")
    held = [weakref.ref(x) for x in (tok, dY, g, coef)]
    opt.step([adamw.TokenGrad(tok, dY), g], 0.01, coef=coef)
    del tok, dY, g, coef
    assert all(r() is None for r in held)
    opt.close()


@pytest.mark.gpu
def test_a_stream_of_another_device():
    class Other:
        device, cuda_stream = torch.device("cuda", 1), 0

    opt = adamw.AdamW([torch.ones(9)], 2, device="cuda:0", outer=lordo.OUTER_AVG)
    g = torch.ones(2, 9, device="cuda:0")
    for call in (lambda: opt.step([g], 0.1, stream=Other()), lambda: opt.outer_step(stream=Other()), lambda: opt.poll_status(stream=Other()),
                 lambda: opt.clear_status(stream=Other())):
        with pytest.raises(ValueError, match="stream"):
            call()
    assert opt.counters() == [0, 0] and (opt.W[0] == 1).all()
    opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("scope", [0, 1])
@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_clip_coefficient_of_a_nan(scope, tokens, dt):
    """min(1, rho / (norm + 1e-6)) of a NaN is NaN, not 1: a NaN does not turn clipping off for the rest of its norm. Of an infinity it is 0."""
    K, shapes = 3, [(40, 24), (300,), (5,)]
    for bad, want in ((float("nan"), float("nan")), (float("inf"), 0.0)):
        opt = group(shapes, K, 1, g_dtype=DT[dt], clip_rho=1.0, clip_scope=scope, tables={0: 30} if tokens else None)
        G = gradients(shapes, K, 1, dt)
        tok = torch.arange(30, device="cuda").repeat(K, 1)
        dY = gradients([(30, 24)], K, 2, dt)[0]
        G64 = [ref.table_grad(tok.cpu().numpy(), ref.to64(dY), 40, 1.0).reshape(K, -1) if tokens else ref.to64(G[0]).reshape(K, -1), ref.to64(G[1]), ref.to64(G[2])]
        coef = ref.clip(G64, 1.0, scope)
        (dY if tokens else G[0])[1, 7, 3] = bad
        opt.step([adamw.TokenGrad(tok, dY) if tokens else G[0]] + G[1:], 0.01)
        got = ref.to64(opt.clip_coefficients())
        hit = np.zeros((3, K), bool)
        hit[slice(0, 3) if scope == 0 else 0, 1] = True
        assert np.array_equal(got[hit], np.full(hit.sum(), want), equal_nan=True)
        assert (np.abs(got - coef)[~hit] <= COEF * coef[~hit]).all()
        assert opt.poll_status() == lordo.FLAG_NONFINITE_GRAD
        opt.close()


@pytest.mark.gpu
@pytest.mark.parametrize("size", [6e18, 1e20, 1e36])
@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_norm_of_gradients_whose_squares_pass_fp32(size, tokens, dt):
    """The sum of squares of a finite gradient is a finite fp64 number: its coefficient is the definition's, and no flag is set. Tokens are all
    different and the scale is 1, so that a row's sum is the row."""
    K, V, d = 2, 2100, 40
    shapes = [(V, d), (9,)]
    opt = group(shapes, K, 1, g_dtype=DT[dt], clip_rho=0.5, tables={0: V} if tokens else None)
    G = gradients(shapes, K, 1, dt, std=1.0)
    G[0] = (G[0].float() * size / G[0].float().abs().max()).to(DT[dt])
    coef = ref.clip([ref.to64(x).reshape(K, -1) for x in G], 0.5)
    opt.step([adamw.TokenGrad(torch.arange(V, device="cuda").repeat(K, 1), G[0]) if tokens else G[0], G[1]], 0.01)
    assert (np.abs(ref.to64(opt.clip_coefficients()) - coef) <= COEF * coef).all()
    assert opt.poll_status() == 0 and torch.isfinite(opt.W[0]).all()
    opt.close()


@pytest.mark.gpu
def test_squares_of_rows_summed_by_token_are_widened_row_by_row():
    """Sums of squares of a table's rows, 32 rows of a window one after another: one row of size 1 (its columns' squares are exact in any order), then
    31 whose squares are 2^-26 each. Added to the first in fp32, each of them would be lost; here they are 31 2^-26 of the norm's square,
    of which a coefficient with a rounding of 2^-24 and a root keeps all but 2^-23."""
    V, d = 32, 8
    opt = adamw.AdamW([torch.zeros(V, d)], 1, clip_rho=1e-3, tables={0: V})
    dY = torch.full((1, V, d), 2.0 ** -13, device="cuda")
    dY[0, 0] = 1.0
    opt.step([adamw.TokenGrad(torch.arange(V, device="cuda").view(1, V), dY)], 0.0)
    norm = (8 * (1 + 31 * 2.0 ** -26)) ** 0.5
    assert abs(float(opt.clip_coefficients()[0, 0].double()) / (1e-3 / (norm + 1e-6)) - 1) <= 2.0 ** -23
    opt.close()


def test_eps_below_the_normal_numbers(lib):
    """In 8 bits the quotient is taken by a reciprocal that takes subnormal numbers for 0: an element without a gradient would be 0 times infinity."""
    tensors = (lordo._Tensor * 1)(lordo._Tensor(100, 0, 0, 0.0))

    def query(states, eps):
        cfg = lordo._AdamWConfig(1, tensors, 2, 0, 0, states, 0.999, eps, 0.0, 0, 0, 0, 0, 0, 1.0, 0.0, 0)
        out = C.c_size_t(0)
        return lib.lordo_adamw_query_workspace(C.byref(cfg), C.byref(out))

    assert query(1, 1e-39) == 1 and query(1, 2.0 ** -127) == 1 and query(1, 2.0 ** -126) == 0 and query(1, 1e-8) == 0
    assert query(0, 1e-39) == 0 and query(0, 1e-50) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("states,eps", [("f32", 1e-39), ("f32", 2.0 ** -126), ("8bit", 2.0 ** -126)])
def test_elements_without_a_gradient_at_the_least_eps(states, eps):
    opt = adamw.AdamW([torch.ones(600)], 1, states=states, eps=eps)
    g = torch.zeros(1, 600, device="cuda")
    g[0, ::7] = 1.0
    opt.step([g], 0.5)
    assert (opt.W[0][g == 0] == 1.0).all()
    assert ((opt.W[0][g != 0] - 0.5).abs() <= 0.5 * 40 * HALF["f32"]).all()  # half of an update of 1, see above
    opt.close()


@pytest.mark.gpu
def test_parameters_as_initial_weights():
    """W0 may be a module's parameters: the group's arrays are no part of their graph."""
    first = torch.nn.Parameter(torch.randn(6, 4))
    opt = adamw.AdamW([first], 2, outer=lordo.OUTER_AVG)
    low = lordo.Lordo([(32, 32, 8)], 2, 1, [torch.nn.Parameter(torch.randn(32, 32))])
    assert torch.equal(opt.W[0][1].cpu(), first.detach())
    for x in list(opt.storage.values()) + opt.W + low.W:
        assert not x.requires_grad and x.grad_fn is None
    opt.close(), low.close()


def _bits16(key, n):
    """ref.random16's bits on the GPU, in 64-bit integers that wrap."""
    signed = lambda x: x - (1 << 64) if x >> 63 else x
    shift = lambda x, s: x ^ ((x >> s) & ((1 << (64 - s)) - 1))
    x = torch.arange(1, n // 4 + 1, device="cuda", dtype=torch.int64) * signed(0x9E3779B97F4A7C15) + signed(key)
    x = shift(shift(x, 30) * signed(0xBF58476D1CE4E5B9), 27) * signed(0x94D049BB133111EB)
    x = shift(x, 31)
    return torch.stack([(x >> s) & 0xFFFF for s in (0, 16, 32, 48)], dim=1).view(-1)


@pytest.mark.gpu
@pytest.mark.parametrize("w", ["f32", "bf16"])
def test_codes_are_those_of_separately_rounded_moments(w):
    """m's 8-bit codes, every one, are those of b1 m, a1 g and their sum each rounded to fp32 (the kernel forms pairs of them in one instruction, and a
    compiler may fuse a product with the sum that takes it: the codes would depend on it). Codes of normal E4M3 numbers are compared: their rounding
    is exact in fp32. 2^25 elements and three steps are enough to tell: the fused form has other codes."""
    from oracle import lordo_oracle as lo
    pow2 = lambda e: ((e.long() + 1023) << 52).view(torch.float64)
    n, b1, a1 = 2 ** 25, torch.tensor(0.9, device="cuda"), torch.tensor(1.0 - 0.9, dtype=torch.float64).float().cuda()
    opt = adamw.AdamW([torch.zeros(n, dtype=DT[w])], 1, states="8bit", seed=13)
    coef, gen, fused_differ = torch.full((1,), 0.7, device="cuda"), torch.Generator(device="cuda").manual_seed(1), 0
    opt.m[0].copy_(torch.randn(n, device="cuda", generator=gen).mul_(60.0).clamp_(-255.0, 255.0))
    opt.v[0].copy_(torch.rand(n, device="cuda", generator=gen).mul_(200.0).add_(20.0))
    opt.ms[0].view(torch.uint8).fill_(127 - 9)
    opt.vs[0].view(torch.uint8).fill_(127 - 9)
    for s in range(1, 4):
        g = torch.randn(1, n, device="cuda", generator=gen).mul_(0.5).to(DT[w])
        m0 = (opt.m[0].float().view(-1, 256) * opt.ms[0].float().view(-1, 1)).view(-1)
        opt.step([g], 0.01, 0.9, coef=coef)
        z = g[0].float() * coef
        key = lo.mix64_int((lo.stream_key(13, 3, 0, s, 0) + lo._GOLDEN) & lo._MASK)
        u = _bits16(key, n)
        assert np.array_equal(u[:1000].cpu().numpy(), ref.random16(13, 3, s, 0, 1000))

        def codes(m):
            a = m.double().abs()
            e = torch.frexp(a.view(-1, 256).amax(dim=1)).exponent - 8
            t = a * pow2(-e.repeat_interleave(256))
            step = pow2(torch.frexp(t).exponent.clamp(min=-5) - 4)
            return torch.copysign((t / step + (u.double() + 0.5) / 65536).floor() * step, m.double()), e, t >= 2.0 ** -6

        q, e, normal = codes(b1 * m0 + a1 * z)
        assert torch.equal(opt.ms[0].view(torch.uint8).view(-1).int(), e + 127)
        assert torch.equal(opt.m[0].view(-1).double()[normal], q[normal])
        other = codes(((b1 * m0).double() + a1.double() * z.double()).float())[0]
        fused_differ += int((other != q)[normal].sum())
    assert fused_differ > 0
    opt.close()


@pytest.mark.gpu
def test_moments_in_32_bits_are_rounded_operation_by_operation():
    n = 2 ** 20 + 3
    opt = adamw.AdamW([torch.zeros(n)], 2, beta2=0.99)
    f32 = lambda x: torch.tensor(x, dtype=torch.float64).float().cuda()
    b1, a1, b2, a2 = f32(0.9), f32(1.0 - 0.9), f32(0.99), f32(1.0 - 0.99)
    coef, m, v = torch.tensor([0.7, 0.3], device="cuda"), torch.zeros(2, n, device="cuda"), torch.zeros(2, n, device="cuda")
    for s in range(3):
        g = gradients([(n,)], 2, s, "f32")[0]
        opt.step([g], 0.01, 0.9, coef=coef)
        z = g * coef.view(2, 1)
        m, v = b1 * m + a1 * z, b2 * v + (a2 * z) * z
        assert torch.equal(opt.m[0], m) and torch.equal(opt.v[0], v)
    opt.close()
