"""event_attention and its gradients against the 64-bit formulas, each value within
the bound that its roundings allow (tests/train_ref.py)."""
import numpy as np
import pytest
import torch

from paper_2607_28940_amd import transx as T
from tests import train_ref as F
from tests.parity_util import log

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    torch.cuda.set_device(0)


def _off(L, first=0):
    return (first + np.concatenate([[0], np.cumsum(L)])).astype(np.int64)


def _where(users, k_first=0, q_first=0):
    """users: [(keys, [(rows, prefix), ...]), ...]"""
    ev = [e for _, es in users for e in es]
    return (_off([k for k, _ in users], k_first), _off([len(es) for _, es in users]), _off([r for r, _ in ev], q_first),
            np.array([p for _, p in ev], dtype=np.int64))


def _inputs(dt, where, H, G, dh, seed=0, logits=1.0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda n, heads, s=1.0: (torch.randn((n, heads, dh), generator=gen) * s).to(dt).cuda()
    N, M = int(where[0][-1]), int(where[2][-1])
    return r(M, H, logits), r(N, G), r(N, G), r(M, H)


def _step(q, k, v, do, where, **kw):
    out, lse = T.event_attention(q, k, v, *where, **kw)
    dq, dk, dv = T.event_attention_backward(do, q, k, v, out, lse, *where, **kw)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _compare(dt, where, H, G, dh, seed=0, **kw):
    q, k, v, do = _inputs(dt, where, H, G, dh, seed, **kw)
    return F.check(_step(q, k, v, do, where), F.attention(q, k, v, F.events(*where), dout=do))


RAGGED = [(130, [(5, 0), (70, 64), (1, 65), (33, 130)]), (1, [(1, 1)]), (64, [(128, 64)]), (0, [(3, 0)]), (40, []),
          (257, [(0, 7), (129, 256), (2, 1), (0, 0), (64, 129)]), (0, []), (63, [(200, 63), (10, 31)])]


@pytest.mark.parametrize("H,G", [(2, 2), (4, 1)])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ragged_users(dtype, dh, H, G):
    """Prefixes and lengths around the tiles, empty prefixes, events and users, prefixes out of order."""
    log(f"event {dtype} d_h {dh} heads {H}/{G}: {_compare(DT[dtype], _where(RAGGED), H, G, dh, seed=dh)}")


@pytest.mark.parametrize("dtype,dh", [("f32", 32), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("users", [
    [(1500, [(1, 1500)])],                                      # a single token
    [(900, [(3, 900)]), (1, [(1, 1)]), (2000, [(20, 1999)])],   # few rows: keys divided
    [(70, [(1500, 70)]), (5, [(300, 4)])],                      # few keys: queries divided
    [(700, [(90, 100 * t + 100) for t in range(7)])],
])
def test_few_rows_or_few_keys(dtype, dh, users):
    log(f"event {dtype} d_h {dh}: {_compare(DT[dtype], _where(users), 2, 1, dh, seed=7, logits=2.0)}")


def test_many_small_users():
    r = np.random.default_rng(3)
    users = [(int(r.integers(0, 30)), []) for _ in range(700)]
    users = [(n, [(int(r.integers(0, 4)), int(r.integers(0, n + 1))) for _ in range(int(r.integers(0, 4)))])
             for n, _ in users]
    _compare(torch.bfloat16, _where(users), 2, 2, 32, seed=1)


@pytest.mark.parametrize("dtype,dh", [("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("-inf")])
def test_keys_past_every_prefix_are_not_read(dtype, dh, bad):
    """Rows that an event does not see may hold anything, within a tile and past it."""
    dt = DT[dtype]
    where = _where([(200, [(40, 50), (30, 100), (9, 0)]), (100, [(50, 70)])])
    q, k, v, do = _inputs(dt, where, 2, 2, dh, seed=11)
    clean = _step(q, k, v, do, where)
    for x in (k, v):
        x[100:200], x[270:300] = bad, bad   # past the longest prefix of each user
    got = _step(q, k, v, do, where)
    assert all(torch.equal(got[n], clean[n]) for n in got)
    # a value row seen by the second event alone
    v[60] = bad
    got = _step(q, k, v, do, where)
    keep = torch.ones(129, dtype=torch.bool, device="cuda")
    keep[40:70] = False
    assert torch.equal(got["out"][keep], clean["out"][keep]) and torch.equal(got["dq"][keep], clean["dq"][keep])
    assert not torch.isfinite(got["out"][40:70]).any()
    # queries and gradients of an event with an empty prefix touch no key
    v[60] = 0.5
    base = _step(q, k, v, do, where)
    q[70:79], do[70:79] = bad, bad
    got = _step(q, k, v, do, where)
    assert torch.equal(got["dk"], base["dk"]) and torch.equal(got["dv"], base["dv"])
    assert bool((got["out"][70:79] == 0).all()) and bool((got["dq"][70:79] == 0).all())


def test_strides_and_rows_outside():
    users = [(90, [(20, 60), (50, 90)]), (33, [(7, 33)])]
    where = _where(users, k_first=4, q_first=9)
    q, k, v, do = _inputs(torch.bfloat16, where, 4, 2, 64, seed=13)
    pad = lambda x: torch.cat([x, torch.full_like(x[:6], float("nan"))])
    q, k, v, do = map(pad, (q, k, v, do))
    q[:9], do[:9], k[:4], v[:4] = (float("nan"),) * 4
    kv = torch.stack([k, v], 2)          # key and value of a head side by side
    wide = torch.stack([q, do], 1)
    out, lse = torch.full_like(q, 5.0), torch.full((4, q.shape[0]), 5.0, device="cuda")
    T.event_attention(wide[:, 0], kv[:, :, 0], kv[:, :, 1], *where, out=out, lse=lse)
    dkv, dq = torch.full_like(kv, 5.0), torch.full_like(q, 5.0)
    T.event_attention_backward(wide[:, 1], wide[:, 0], kv[:, :, 0], kv[:, :, 1], out, lse, *where, dq=dq,
                               dk=dkv[:, :, 0], dv=dkv[:, :, 1])
    M, N = int(where[2][-1]), int(where[0][-1])
    inner = (where[0] - 4, where[1], where[2] - 9, where[3])
    want = F.attention(q[9:M], k[4:N], v[4:N], F.events(*inner), dout=do[9:M])
    F.check({"out": out[9:M], "lse": lse[:, 9:M], "dq": dq[9:M], "dk": dkv[4:N, :, 0], "dv": dkv[4:N, :, 1]}, want)
    for x, a, b in ((out, 9, M), (dq, 9, M), (dkv, 4, N), (lse.t(), 9, M)):
        assert bool((x[:a] == 5.0).all()) and bool((x[b:] == 5.0).all())


def test_broadcast_heads_and_scale():
    """Key heads read through a stride of 0, and a scale of the caller's."""
    where = _where([(100, [(30, 100), (40, 80)])])
    q, k, v, do = _inputs(torch.bfloat16, where, 4, 1, 64, seed=17)
    ke, ve = k.expand(-1, 4, -1), v.expand(-1, 4, -1)
    out, lse = T.event_attention(q, ke, ve, *where, scale=0.3)
    dk, dv = (torch.empty(100, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dq, _, _ = T.event_attention_backward(do, q, ke, ve, out, lse, *where, scale=0.3, dk=dk, dv=dv)
    want = F.attention(q, ke, ve, F.events(*where), scale=float(np.float32(0.3)), dout=do)
    F.check({"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, want)
    shared = _step(q, k, v, do, where, scale=0.3)
    assert torch.equal(shared["out"], out) and torch.equal(shared["dq"], dq)


def test_offsets_past_32_bits():
    """Rows more than 2^32 bytes and 2^31 elements from a tensor's start."""
    dt, H, dh = torch.bfloat16, 2, 64
    M = 70
    row = 1 << 22                              # elements between rows: 8 MiB
    big = torch.zeros(700 * row, dtype=dt, device="cuda")
    far = big.as_strided((700, H, dh), (row, dh, 1))
    where = (np.array([600, 690]), np.array([0, 2]), np.array([0, 30, M]), np.array([50, 90]))
    gen = torch.Generator().manual_seed(23)
    k, v = ((torch.randn(90, H, dh, generator=gen)).to(dt).cuda() for _ in range(2))
    q, do = ((torch.randn(M, H, dh, generator=gen)).to(dt).cuda() for _ in range(2))
    far[600:690] = k
    vfar = torch.zeros(690, H, dh, dtype=dt, device="cuda")
    vfar[600:] = v
    out, lse = T.event_attention(q, far[:690], vfar, *where)
    dk, dv = torch.zeros_like(vfar), torch.zeros_like(vfar)
    dq, _, _ = T.event_attention_backward(do, q, far[:690], vfar, out, lse, *where, dk=dk, dv=dv)
    near = (where[0] - 600,) + where[1:]
    same = _step(q, k, v, do, near)
    assert torch.equal(out, same["out"]) and torch.equal(dq, same["dq"])
    assert torch.equal(dk[600:], same["dk"]) and torch.equal(dv[600:], same["dv"])


def test_gradients_by_differences():
    where = _where([(30, [(9, 12), (14, 30)]), (8, [(5, 8)])])
    q, k, v, do = _inputs(torch.float32, where, 2, 1, 32, seed=31)
    got = _step(q, k, v, do, where)
    gen = torch.Generator().manual_seed(4)
    f = lambda *a: float((F.attention(*a, F.events(*where))["out"][0] * do.cpu().double()).sum())
    base = [x.cpu().double() for x in (q, k, v)]
    for i, n in enumerate(("dq", "dk", "dv")):
        d = torch.randn(base[i].shape, generator=gen, dtype=torch.float64)
        h = 1e-4
        up, down = ([b + s * h * d if j == i else b for j, b in enumerate(base)] for s in (1, -1))
        # central differences are off by h^2 / 6 of a third derivative of order 10^2 here
        want, have = (f(*up) - f(*down)) / (2 * h), float((got[n].cpu().double() * d).sum())
        assert abs(want - have) <= 2e-5 * (1 + abs(want)), (n, want, have)


def test_graphs_of_divided_blocks():
    """Two captured steps (few rows: divided keys and joins) and eager ones in turn."""
    where = _where([(3000, [(4, 1000), (9, 3000)]), (500, [(1, 400)])])
    q, k, v, do = _inputs(torch.bfloat16, where, 4, 2, 128, seed=19)
    first = _step(q, k, v, do, where)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = _step(q, k, v, do, where)
        graphs.append((g, res))
    for _ in range(3):
        for g, res in graphs:
            for x in res.values():
                x.fill_(3.0)
            g.replay()
        _step(q * 2, k, v, do, where)
        torch.cuda.synchronize()
        assert all(torch.equal(first[n], res[n]) for _, res in graphs for n in first)


FEW_ROWS = [(4500, [(33, 4500), (1, 4097)])]                         # long keys, divided blocks
MANY = [(1 + 37 * u % 150, [(1 + 13 * u % 70, 0 if u % 9 == 0 else 1 + u % (1 + 37 * u % 150)), (u % 3, 1)])
        for u in range(260)]


@pytest.mark.parametrize("users", [FEW_ROWS, MANY], ids=["few_rows", "many"])
@pytest.mark.parametrize("H,G", [(4, 2), (6, 1), (8, 1), (12, 3)])
@pytest.mark.parametrize("dtype,dh", [("f32", 32), ("f32", 128), ("bf16", 64), ("bf16", 128)])
def test_heads_that_share_a_block(dtype, dh, H, G, users):
    """2, 6, 8 and 4 query heads a key head: blocks of 64 rows of 2 heads, or of 32 rows of 4."""
    _compare(DT[dtype], _where(users), H, G, dh, seed=H)


@pytest.mark.parametrize("H,G", [(1, 1), (2, 1), (2, 2), (4, 4), (3, 3)])
def test_head_counts_and_many_blocks(H, G):
    """1, 2, 4 and 3 heads (or pairs of heads): how blocks are dealt to the chip, with units left over."""
    users = [(64 * u % 301, [(1 + 17 * u % 200, 64 * u % 301)]) for u in range(530 // H)]
    _compare(torch.bfloat16, _where(users), H, G, 32, seed=3)


def test_more_blocks_than_are_sorted():
    r = np.random.default_rng(5)
    users = [(int(r.integers(0, 9)), []) for _ in range(4500)]
    users = [(n, [(int(r.integers(1, 3)), int(r.integers(0, n + 1)))]) for n, _ in users]
    users[2000] = (300, [(140, 299), (3, 7)])
    _compare(torch.bfloat16, _where(users), 1, 1, 32, seed=2)
