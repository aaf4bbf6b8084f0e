"""Rotary positions on the GPU: the table against extended precision, the rotation bit for
bit against its definition, the write into the 8-bit cache against rotation and append."""
import numpy as np
import pytest
import torch

from paper_2609_17475_amd import jfkv
from tests.kv8_cases import Pair, dtype_of, i32, rows, tables_for

pytestmark = pytest.mark.gpu


def f32(x):
    return torch.tensor(np.asarray(x, np.float32), device="cuda")


def make_table(rng, n, rot, spread=100000):
    """(the table as the library forms it, its positions)."""
    pos = i32(rng.integers(-spread, spread, n))
    freq = f32(np.exp(-rng.uniform(0, 9, rot // 2)))
    table = torch.empty((n, rot // 2, 2), device="cuda")
    jfkv.jf_rope_table(pos, freq, table)
    return table


def turned(x, table, rot, pairs, back=False):
    """The definition: products and sums rounded in fp32 one by one.  x [n][heads][d] on
    the CPU, a table row for each of the n."""
    t = table.cpu()[:, None]
    c, s = t[..., 0], -t[..., 1] if back else t[..., 1]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y = x.float()
    x1, x2 = y[..., a].clone(), y[..., b].clone()
    y[..., a] = x1 * c - x2 * s
    y[..., b] = x2 * c + x1 * s
    return y.to(x.dtype)


# ------------------------------------------------------------------- table
@pytest.mark.parametrize("rot", [2, 6, 64, 130, 256])
@pytest.mark.parametrize("magnitude", [1.0, 1.2079])
def test_table(rot, magnitude):
    rng = np.random.default_rng(rot)
    pos = np.concatenate(([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 262143], rng.integers(-10 ** 6, 10 ** 6, 50),
                          rng.integers(-2 ** 31, 2 ** 31, 50)))
    freq = np.exp(-rng.uniform(0, 12, rot // 2)).astype(np.float32)
    freq[0] = 1.0
    table = torch.full((len(pos) + 1, rot // 2, 2), 7.0, device="cuda")
    jfkv.jf_rope_table(i32(pos), f32(freq), table[:-1], magnitude)
    x = np.longdouble
    angle = pos.astype(x)[:, None] * freq.astype(x)  # exact: 32 and 24 bits in 64
    # (pi in extended precision is good to 2^-64, an angle of 2^31 to 2^-33 after its turns)
    m = x(np.float32(magnitude))
    want = np.stack((np.cos(angle), np.sin(angle)), 2) * m
    got = table.cpu().numpy().astype(x)
    # one rounding to fp32; the series' rests, sums in 64 bits, pi's digits: below 2^-32
    assert np.all(np.abs(got[:-1] - want) <= np.abs(want) * 2.0 ** -24 + 2.0 ** -32)
    assert np.all(got[-1] == 7.0)


# ---------------------------------------------------------------- rotation
CASES = [  # tokens, hq, hk, d, rot, pairs, bf16
    (1, 1, 0, 2, 2, False, False),
    (1, 4, 1, 128, 128, False, False),
    (3, 32, 8, 128, 128, False, True),
    (7, 24, 4, 256, 64, True, True),
    (5, 3, 2, 64, 64, True, False),
    (33, 5, 3, 80, 20, False, False),
    (9, 2, 1, 96, 72, True, False),
    (4, 7, 3, 64, 2, True, True),
    (6, 3, 1, 128, 126, False, True),
    (2, 1, 3, 10, 6, False, False),
    (2, 2, 2, 300, 150, True, True),
    (1, 1, 1, 2048, 1030, False, False),
    (5000, 2, 1, 64, 32, False, True),
    (4097, 1, 1, 66, 66, False, False),
]


@pytest.mark.parametrize("n,hq,hk,d,rot,pairs,bf16", CASES)
@pytest.mark.parametrize("form", ["apart", "packed", "inplace", "odd", "back"])
def test_rotation_is_bit_exact(n, hq, hk, d, rot, pairs, bf16, form):
    rng = np.random.default_rng(n + d + rot)
    table = make_table(rng, n, rot)
    t = dtype_of(bf16)
    back = form == "back"
    gap = {"packed": hk + 1, "odd": 0}.get(form, 0)  # (heads of the row that nobody rotates)
    width = (hq + hk + gap) * d + (3 if form == "odd" else 0)
    off = 1 if form == "odd" else 0
    x = torch.from_numpy(rng.standard_normal((n, width)) * 4).to(t)

    def parts(z):
        return (z[:, off:off + hq * d].view(n, hq, d),
                z[:, off + hq * d:off + (hq + hk) * d].view(n, hk, d))

    q, k = parts(x)
    dev = x.cuda()
    dq, dk = parts(dev)
    to = dev if form == "inplace" else torch.full((n, width + 8), 3.0, dtype=t, device="cuda")[:, :width]
    oq, ok = parts(to)
    rope = jfkv.Rope(table, pairs=pairs)
    if hk:
        jfkv.jf_rope_rotate(rope, dq, oq, dk, ok, transpose=back)
    else:
        jfkv.jf_rope_rotate(rope, dq, oq, transpose=back)
    assert torch.equal(oq.cpu().view(torch.int16), turned(q, table, rot, pairs, back).view(torch.int16))
    if hk:
        assert torch.equal(ok.cpu().view(torch.int16), turned(k, table, rot, pairs, back).view(torch.int16))
    rest = to.cpu().clone()
    was = x.clone() if form == "inplace" else torch.full_like(rest, 3.0)
    rest[:, off:off + (hq + hk) * d] = 0
    was[:, off:off + (hq + hk) * d] = 0
    assert torch.equal(rest, was)  # nothing else is written
    if form != "inplace":
        assert torch.equal(dev.cpu(), x)


@pytest.mark.parametrize("pairs", [False, True])
def test_keys_alone_and_rows_of_a_shared_table(pairs):
    rng = np.random.default_rng(3)
    table = make_table(rng, 17, 48)
    index = np.concatenate((rng.integers(0, 17, 60), [-5, 17, 2 ** 31 - 1, -2 ** 31]))
    x = torch.from_numpy(rng.standard_normal((64, 3, 64))).half()
    y = torch.empty_like(x, device="cuda")
    jfkv.jf_rope_rotate(jfkv.Rope(table, rows=i32(index), pairs=pairs), None, None, x.cuda(), y)
    want = turned(x, table[torch.from_numpy(np.clip(index, 0, 16)).cuda()], 48, pairs)
    assert torch.equal(y.cpu(), want)


def test_special_values():
    """Infinities and NaN stay in their pair; zero angles leave rows as they are."""
    table = torch.zeros((2, 4, 2), device="cuda")
    table[0, :, 0] = 1.0
    table[1] = f32([[0.6, 0.8]] * 4)
    x = torch.tensor([[[1.0, 2, 3, 4, -5, 6, 7, 8]], [[float("inf"), 2, float("nan"), 4, 5, 6, 7, 8]]],
                     dtype=torch.float16)
    y = torch.empty_like(x, device="cuda")
    jfkv.jf_rope_rotate(jfkv.Rope(table), x.cuda(), y)
    y = y.cpu()
    assert torch.equal(y[0], x[0])
    assert y[1, 0, 0] == float("inf") and y[1, 0, 4] == float("inf")
    assert torch.isnan(y[1, 0, [2, 6]]).all()
    assert torch.isfinite(y[1, 0, [1, 3, 5, 7]]).all()
    big = torch.full((1, 1, 8), 65504.0, dtype=torch.float16, device="cuda")
    table[0] = f32([[0.8, 0.6]] * 4)
    jfkv.jf_rope_rotate(jfkv.Rope(table), big, big)
    assert torch.isinf(big[0, 0, 4:]).all() and torch.isfinite(big[0, 0, :4]).all()


@pytest.mark.parametrize("pairs,rot,d", [(False, 64, 64), (True, 48, 64), (False, 6, 10)])
def test_gradient(pairs, rot, d):
    """d loss / d x_j for loss = sum of g y(x): the transposed rotation of g against
    the formula in 64 bits, and against differences, the loss of unit steps (which for a
    linear map are exact up to roundings)."""
    rng = np.random.default_rng(d)
    table = make_table(rng, 1, rot)
    g = torch.from_numpy(rng.standard_normal((1, 1, d))).half()
    grad = torch.empty_like(g, device="cuda")
    jfkv.jf_rope_rotate(jfkv.Rope(table, pairs=pairs), g.cuda(), grad, transpose=True)
    grad = grad.cpu().double().numpy()[0, 0]
    t, gg = table.cpu().double().numpy()[0], g.double().numpy()[0, 0]
    want = gg.copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
        c, s = t[i]
        want[a], want[b] = c * gg[a] + s * gg[b], c * gg[b] - s * gg[a]
    scale = np.abs(gg).max() * 2
    # two products and a sum in fp32, the rounding to fp16
    assert np.all(np.abs(grad - want) <= np.abs(want) * 2.0 ** -11 + scale * 2.0 ** -22 + 2.0 ** -25)
    eye = torch.eye(d, dtype=torch.float16, device="cuda")[:, None].contiguous()
    step = torch.empty_like(eye)
    rope = jfkv.Rope(table, rows=torch.zeros(d, dtype=torch.int32, device="cuda"), pairs=pairs)
    jfkv.jf_rope_rotate(rope, eye, step)
    loss = step[:, 0].cpu().double().numpy() @ gg  # two entries of each row, rounded to fp16
    assert np.all(np.abs(grad - loss) <= np.abs(grad) * 2.0 ** -11 + scale * 2.0 ** -11 + 2.0 ** -24)


def test_rows_beyond_32_bits():
    """A wide projection's last rows lie behind 2^31 elements."""
    n, d, stride = 33000, 64, 65544  # 2.16e9 elements
    wide = torch.zeros(n * stride, dtype=torch.float16, device="cuda")
    x = wide.as_strided((n, 1, d), (stride, d, 1))
    rng = np.random.default_rng(1)
    table = make_table(rng, n, d)
    x[-3:] = torch.from_numpy(rng.standard_normal((3, 1, d))).half().cuda()
    want = turned(x[-3:].cpu(), table[-3:], d, False)
    jfkv.jf_rope_rotate(jfkv.Rope(table), x, x)
    assert torch.equal(x[-3:].cpu(), want)
    assert not x[:-3].any()


def test_refusals_of_the_binding():
    t = torch.zeros((4, 8, 2), device="cuda")
    x = torch.zeros((4, 2, 16), dtype=torch.float16, device="cuda")
    rope = jfkv.Rope(t)
    for q, o in ((x.float(), x.float()), (x, x.bfloat16()), (x.cpu(), x), (x, x[:3]), (x, None),
                 (x.transpose(0, 1), x.transpose(0, 1)), (x[..., ::2], x[..., ::2]),
                 (x[0], x[0])):
        with pytest.raises(ValueError):
            jfkv.jf_rope_rotate(rope, q, o)
    with pytest.raises(ValueError):
        jfkv.jf_rope_rotate(jfkv.Rope(t, rows=torch.zeros(3, dtype=torch.int32, device="cuda")), x, x)
    with pytest.raises(ValueError):
        jfkv.jf_rope_rotate(rope, x, x, x[:2], x[:2])
    with pytest.raises(ValueError):
        jfkv.Rope(t[..., 0])
    with pytest.raises(jfkv.JfError):
        jfkv.jf_rope_rotate(jfkv.Rope(t[:3]), x, x)  # fewer rows than tokens
    with pytest.raises(jfkv.JfError):
        jfkv.jf_rope_rotate(rope, x[:, :, :8].contiguous(), x[:, :, :8].contiguous())  # rot_dim > d


# ------------------------------------------------------- into the 8-bit cache
@pytest.mark.parametrize("P,hkv,gq,d,block,rot,pairs,bf16,lens,prefix", [
    (64, 1, 4, 64, 16, 64, False, False, [1], 0),
    (64, 2, 1, 64, 32, 16, False, True, [130, 1, 0, 64], 0),
    (128, 3, 2, 128, 16, 128, True, False, [5, 200, 33], 0),
    (256, 2, 4, 128, 64, 128, False, False, [300, 77], 0),
    (256, 1, 6, 256, 128, 64, True, True, [257, 600], 0),
    (64, 2, 3, 256, 64, 256, False, False, [64, 63, 65], 0),
    (128, 2, 2, 128, 128, 48, False, False, [100, 28, 129], 51),
    (64, 1, 8, 128, 16, 80, True, True, [1, 1, 17, 40, 3], 23),
])
@pytest.mark.parametrize("packed", [False, True])
def test_rope_append_is_rotate_then_append(P, hkv, gq, d, block, rot, pairs, bf16, lens, prefix, packed):
    rng = np.random.default_rng(P + d + block + len(lens))
    total = [n + prefix for n in lens]
    pages = sum(-(-max(n, 1) // P) for n in total) + 2
    p = Pair(P, hkv, d, block, pages, bf16)
    tables, _ = tables_for(rng, P, total, pages)
    if prefix:
        p.fill(rng, [prefix] * len(lens), tables)
    n, hq = sum(lens), hkv * gq
    k, v, q = rows(rng, n, hkv, d, bf16, 3.0), rows(rng, n, hkv, d, bf16), rows(rng, n, hq, d, bf16)
    table = make_table(rng, n + 5, rot)
    index = rng.integers(0, n + 5, n)
    rope = jfkv.Rope(table, rows=i32(index), pairs=pairs)
    dk, dv, dq = k.cuda(), v.cuda(), q.cuda()
    if packed:
        x = torch.cat((dq, dk, dv), 1)
        dq, dk, dv = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    out = torch.full((n + 1, hq, d), 3.0, dtype=q.dtype, device="cuda")
    cu = np.cumsum([0] + lens).tolist()
    start = [prefix] * len(lens)
    jfkv.jf_kv8_rope_append(p.gpu, rope, dk, dv, i32(cu), i32(start), i32(tables), q=dq, q_out=out[:n])
    tab = table[torch.from_numpy(index).cuda()]
    rk = turned(k, tab, rot, pairs)
    p.host.append(rk.double().numpy(), v.double().numpy(), cu, start, tables)
    assert not p.differing()
    assert torch.equal(out[:n].cpu().view(torch.int16), turned(q, tab, rot, pairs).view(torch.int16))
    assert (out[n] == 3.0).all()
    # without queries: the same cache
    p2 = Pair(P, hkv, d, block, pages, bf16)
    for name in ("k_codes", "k_exps", "v_codes", "v_exps"):
        getattr(p2.gpu, name).copy_(getattr(p.gpu, name))
    jfkv.jf_kv8_rope_append(p2.gpu, rope, dk, dv, i32(cu), i32(start), i32(tables))
    for name in ("k_codes", "k_exps", "v_codes", "v_exps"):
        assert torch.equal(getattr(p2.gpu, name), getattr(p.gpu, name))


def test_rope_append_in_place_and_skipped_rows():
    """Keys without a page are skipped, their queries are rotated all the same."""
    rng = np.random.default_rng(8)
    p = Pair(64, 2, 64, 16, 3, True)
    tables = np.array([[1, -1], [2, 99]], np.int32)
    cu, start = [0, 70, 140], [20, 10]
    k, v, q = (rows(rng, 140, h, 64, True) for h in (2, 2, 4))
    table = make_table(rng, 140, 32)
    dq = q.cuda()
    jfkv.jf_kv8_rope_append(p.gpu, jfkv.Rope(table), k.cuda(), v.cuda(), i32(cu), i32(start),
                            i32(tables), q=dq, q_out=dq)
    p.host.append(turned(k, table, 32, False).double().numpy(), v.double().numpy(), cu, start, tables)
    assert not p.differing()
    assert torch.equal(dq.cpu(), turned(q, table, 32, False))


def test_captured_and_on_another_stream():
    """Table, rotation and write captured in a graph, replayed with new positions and rows."""
    rng = np.random.default_rng(9)
    B, hq, hkv, d = 3, 4, 2, 128
    p = Pair(64, hkv, d, 16, 8, False)
    tables = i32(np.array([[0, 5], [3, 1], [2, 7]], np.int32))
    freq = f32(np.exp(-rng.uniform(0, 9, d // 2)))
    pos, start = i32([0, 0, 0]), i32([0, 0, 0])
    x = torch.zeros((B, hq + 2 * hkv, d), dtype=torch.float16, device="cuda")
    table = torch.empty((B, d // 2, 2), device="cuda")
    q_out, k_out = torch.empty((B, hq, d), dtype=torch.float16, device="cuda"), torch.empty_like(x[:, :hkv]).contiguous()
    cu = i32([0, 1, 2, 3])
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    def step():
        jfkv.jf_rope_table(pos, freq, table)
        rope = jfkv.Rope(table)
        jfkv.jf_rope_rotate(rope, q, q_out, k, k_out)
        jfkv.jf_kv8_rope_append(p.gpu, rope, k, v, cu, start, tables)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for turn in range(4):
        new = torch.from_numpy(rng.standard_normal((B, hq + 2 * hkv, d))).half()
        x.copy_(new)
        at = rng.integers(0, 100000, B)
        pos.copy_(torch.from_numpy(at).int())
        start.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        tab = table.cpu().clone()
        ang = at.astype(np.longdouble)[:, None] * freq.cpu().numpy().astype(np.longdouble)
        want = np.stack((np.cos(ang), np.sin(ang)), 2)
        assert np.all(np.abs(tab.numpy() - want) <= np.abs(want) * 2.0 ** -24 + 2.0 ** -32)
        assert torch.equal(q_out.cpu(), turned(new[:, :hq], tab, d, False))
        rk = turned(new[:, hq:hq + hkv], tab, d, False)
        assert torch.equal(k_out.cpu(), rk)
        p.host.append(rk.double().numpy(), new[:, hq + hkv:].double().numpy(), [0, 1, 2, 3],
                      start.cpu().tolist(), tables.cpu().numpy())
        assert not p.differing()
