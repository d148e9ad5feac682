"""Calls of the microscaled 4-bit operators at the edges of what the header allows."""
import numpy as np
import pytest

import mx_plain

pytestmark = pytest.mark.gpu


def _mx():
    from paper_2106_05373_amd import mx
    return mx


def _bcpnn():
    from paper_2106_05373_amd import bcpnn
    return bcpnn


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def test_a_layer_whose_inputs_broke_their_pairs_is_not_copied():
    """Making a copy waits for the stream, so it reports what training saw of the inputs."""
    import torch
    B = _bcpnn()
    cfg = B.default_config(64, 2, 4, 16, 32, complement_pairs=1)
    pixels = torch.rand(32, 64, generator=_gen(1), device="cuda")
    x = torch.stack([pixels, 1 - pixels], 2).reshape(32, 128).contiguous()
    with B.Layer(cfg) as layer:
        layer.train_batch(x)
        _mx().Layer.of(layer).close()
        x[5, 7] += 0.25
        layer.train_batch(x)
        with pytest.raises(B.BcpnnError, match="EINPUT"):
            _mx().Layer.of(layer)
        with pytest.raises(B.BcpnnError, match="ESTATE"):
            _mx().Layer.of(layer)


def test_every_batch_of_a_layer_of_very_many_hidden_hcus():
    """2^21 hidden HCUs, the most for which 64 rows are a batch."""
    import torch
    B = _bcpnn()
    ho, n = 1 << 21, 64
    cfg = B.default_config(2, 1, ho, 1, n)
    w = torch.randn(2, ho, generator=_gen(1), device="cuda")
    b = torch.randn(ho, generator=_gen(2), device="cuda")
    x = torch.rand(n, 2, generator=_gen(3), device="cuda")
    with _mx().Layer(cfg, None, w, b) as layer:
        y, s = (torch.full((n + 1, ho), 5.0, device="cuda") for _ in range(2))
        for rows in (1, 33, n):
            layer.forward(x[:rows], y[:rows], s[:rows])
            xq = torch.from_numpy(mx_plain.quantized(x[:rows].cpu().numpy())).cuda()
            wq = _mx().dequantize(_mx().quantize(w, rows=False, columns=True)).double().t()
            want = xq @ wq + b.double()
            mag = xq.abs() @ wq.abs() + b.double().abs()
            assert bool(((s[:rows].double() - want).abs() <= mag * mx_plain.sum_bound(2)).all()), rows
            assert bool((y[:rows] == 1.0).all()) and bool((y[rows:] == 5.0).all()) and bool((s[rows:] == 5.0).all())
            y.fill_(5.0)
            s.fill_(5.0)


@pytest.mark.parametrize("in_hcu,in_mcu", [(31, 1), (45, 2), (33, 3), (12, 4)])
def test_predict_with_any_number_of_workspace_rows(in_hcu, in_mcu):
    """Rows of x that start at any alignment of their elements."""
    import torch
    B, mx = _bcpnn(), _mx()
    n_in = in_hcu * in_mcu
    hidden = mx.Layer(B.default_config(in_hcu, in_mcu, 3, 9, 16), None,
                      torch.randn(n_in, 27, generator=_gen(1), device="cuda"), torch.zeros(27, device="cuda"))
    readout = mx.Layer(B.default_config(3, 9, 1, 6, 16), None,
                       torch.randn(27, 6, generator=_gen(2), device="cuda"), torch.zeros(6, device="cuda"))
    x = torch.rand(11, n_in, generator=_gen(3), device="cuda")
    y = torch.empty(11, 27, device="cuda")
    want = torch.empty(11, 1, device="cuda", dtype=torch.int32)
    hidden.forward(x, y)
    readout.readout(y, want)
    for rows in (1, 2, 3, 5, 11):
        got = torch.full((12,), -1, device="cuda", dtype=torch.int32)
        hidden.predict_with(readout, x, torch.empty(rows, 27, device="cuda"), got[:11])
        assert torch.equal(got[:11], want[:, 0]) and got[11] == -1, rows
    hidden.close()
    readout.close()


def _small_network():
    import torch
    from paper_2106_05373_amd.pipeline import Network
    B = _bcpnn()
    net = Network(B.default_config(64, 2, 4, 16, 32, alpha=0.05, seed=3), None, 5)
    x = torch.rand(70, 128, generator=_gen(4), device="cuda")
    target = torch.nn.functional.one_hot(torch.arange(32, device="cuda") % 5, 5).float()
    for _ in range(4):
        net.train_hidden(x[:32])
        net.train_readout(x[:32], target)
    return net, x


def test_quantized_network_writes_every_output_that_a_network_writes():
    import torch
    net, x = _small_network()
    q = net.quantized()
    want = q.predict(x)
    assert want.dtype == torch.int32 and want.shape == (70,)
    room = torch.full((70, 3), -1, device="cuda", dtype=torch.int32)
    outs = [torch.full((70,), -1, device="cuda", dtype=torch.int64), room[:, 1],
            torch.full((70,), -1, dtype=torch.int32), torch.full((70,), -1.0, device="cuda")]
    for out in outs:
        assert net.predict(x, out=out) is out           # (the network itself takes them)
        out.fill_(-1)
        assert q.predict(x, out=out) is out
        assert torch.equal(out.cuda().int(), want)
    assert bool((room[:, 0] == -1).all()) and bool((room[:, 2] == -1).all())
    q.close()
    net.close()


def test_quantized_network_holds_its_workspace_on_its_stream():
    """Every prediction uses it there, whichever stream is current when it is made or called: memory of
    another stream's pool may still be in use by work that this stream does not wait for."""
    import torch
    from paper_2106_05373_amd.pipeline import Network
    B = _bcpnn()
    own = torch.cuda.Stream()
    net = Network(B.default_config(64, 2, 4, 16, 32), None, 5, stream=own)
    q = net.quantized()
    at = q._rows.data_ptr()
    held = [s for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]
    assert len(held) == 1 and held[0]["stream"] == own.cuda_stream
    q.close()
    net.close()


def test_a_layer_on_another_stream_waits_for_its_weights():
    import torch
    B = _bcpnn()
    cfg = B.default_config(100, 2, 3, 40, 32)
    final = torch.randn(200, 120, generator=_gen(1), device="cuda")
    x = torch.rand(32, 200, generator=_gen(2), device="cuda")
    big = torch.randn(8192, 8192, device="cuda")
    w, b = torch.zeros_like(final), torch.zeros(120, device="cuda")
    want = torch.empty(32, 120, device="cuda")
    with _mx().Layer(cfg, None, final, b) as layer:
        layer.forward(x, torch.empty_like(want), want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        big @ big                                       # (milliseconds of work before the weights are written)
    w.copy_(final)
    layer = _mx().Layer(cfg, None, w, b, stream=side)
    got = torch.empty_like(want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        layer.forward(x, torch.empty_like(want), got)
    side.synchronize()
    assert torch.equal(got, want)
    layer.close()


def test_one_long_row_is_quantised_by_row_and_read_back():
    """2^21 pieces of 32 x 256: a launch of 2^29 work-items."""
    import torch
    mx = _mx()
    cols = 1 << 29
    x = torch.zeros(1, cols, device="cuda", dtype=torch.bfloat16)
    ends = torch.cat([torch.arange(64), cols // 2 + torch.arange(64), cols - 64 + torch.arange(64)]).cuda()
    x[0, ends] = torch.randn(192, generator=_gen(1), device="cuda").bfloat16()
    m = mx.quantize(x)
    out = mx.dequantize(m, torch.bfloat16)
    want = mx_plain.quantized(x[:, ends].double().cpu().numpy())
    assert np.array_equal(out[:, ends].double().cpu().numpy(), want)
    out[0, ends] = 0
    assert not bool(out.any())
    with pytest.raises(_bcpnn().BcpnnError):            # 2^24 pieces with the rows filled up to 256
        mx.quantize(x, rows=False, columns=True)


def test_product_of_few_rows_and_very_many_columns():
    """2^32 outputs, of which a work-item stores several: a launch of 2^29."""
    import torch
    mx = _mx()
    m, n = 64, 1 << 26
    a = torch.randn(m, 1, generator=_gen(1), device="cuda")
    b = torch.randn(n, 1, generator=_gen(2), device="cuda").half()
    qa, qb = mx.quantize(a), mx.quantize(b)
    del b
    c = mx.product(qa, qb, dtype=torch.float16)
    av, bv = mx.dequantize(qa), mx.dequantize(qb)
    at = torch.cat([torch.arange(100), n // 2 + torch.arange(100), n - 100 + torch.arange(100)]).cuda()
    want = av @ bv[at].t()                              # one product of 4-bit values: exact
    assert torch.equal(c[:, at], want.half())


# (sizes for each kind of tile, whole and not, several tiles per workgroup among them)
TILES = [(900, 850, 700), (2304, 2560, 300), (2310, 2571, 700), (4352, 4096, 300), (4100, 4203, 700), (4100, 4203, 100)]
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


@pytest.mark.parametrize("dtype", list(HALF_STEP))
@pytest.mark.parametrize("m,n,k", TILES)
def test_tiles_with_bias_scaling_accumulation_and_stride(m, n, k, dtype):
    import torch
    mx, g = _mx(), _gen(m + k)
    T = getattr(torch, dtype)
    a, b = (mx.quantize(torch.randn(r, k, generator=g, device="cuda")) for r in (m, n))
    bias = torch.randn(n, generator=g, device="cuda")
    av, bv = mx.dequantize(a).double(), mx.dequantize(b).double()
    dot, mag = av @ bv.t(), av.abs() @ bv.abs().t()
    for start, alpha, beta in ((0, 1.0, 0.0), (1, 0.375, -0.5), (3, -2.0, 1.0)):
        room = torch.randn(m + 1, n + 5, generator=g, device="cuda").to(T)
        before = room.clone()
        out = room[:m, start:start + n]
        c0 = out.double()
        mx.product(a, b, bias=bias, alpha=alpha, beta=beta, out=out)
        want = alpha * dot + beta * c0 + bias.double()
        size = abs(alpha) * mag + (beta * c0).abs() + bias.double().abs()
        # the sum's bound, then one rounding to the type of a value within it
        bound = size * mx_plain.sum_bound(k) * (1 + HALF_STEP[dtype])
        if dtype != "float32":
            bound = bound + want.abs() * HALF_STEP[dtype] + (2.0 ** -25 if dtype == "float16" else 0.0)
        assert bool(((out.double() - want).abs() <= bound).all()), (start, alpha, beta)
        out.copy_(before[:m, start:start + n])
        assert torch.equal(room, before)                # nothing beside the output changed


@pytest.mark.parametrize("m,n,k", [(30, 500, 5000), (40, 256, 3000), (200, 300, 700), (900, 850, 260), (2304, 2560, 300),
                                   (4100, 4203, 300)])
def test_a_row_of_a_product_does_not_depend_on_the_other_rows(m, n, k):
    import torch
    mx, g = _mx(), _gen(m)
    x, w = (torch.randn(r, k, generator=g, device="cuda") for r in (m, n))
    b = mx.quantize(w)
    c = mx.product(mx.quantize(x), b)
    for row in (0, m // 2, m - 1):
        other = torch.randn(m, k, generator=g, device="cuda") * 100
        other[(row + 1) % m] = float("nan")
        other[row] = x[row]
        assert torch.equal(mx.product(mx.quantize(other), b)[row], c[row]), row


def test_products_of_far_scales():
    """Scales from 2^-126 to 2^125 on both sides, met by zeros and by scales that take them back."""
    import torch
    mx = _mx()
    e = np.array([-120, -60, 0, 60, 120])
    a = np.zeros((20, 320), np.float32)
    b = np.zeros((20, 320), np.float32)
    for i in range(5):
        a[4 * i:4 * i + 4, 64 * i:64 * i + 32] = np.ldexp(1.5, e[i])       # meets the opposite scale: 2.25
        b[4 * i:4 * i + 4, 64 * i:64 * i + 32] = np.ldexp(1.5, -e[i])
        a[4 * i:4 * i + 4, 64 * i + 32] = np.ldexp(1.0, 120)               # meets a zero of a block as large
        b[4 * i:4 * i + 4, 64 * i + 33] = np.ldexp(1.0, 120)
    want, _ = mx_plain.product(mx_plain.quantized(a), mx_plain.quantized(b))
    assert np.array_equal(want[::4, ::4], 72 * np.eye(5))
    for rows in (1, 20, 900):
        at = np.resize(np.arange(20), rows)
        t = torch.from_numpy(a[at]).cuda()
        u = torch.from_numpy(np.resize(b, (900 if rows == 900 else 20, 320))).cuda()
        got = mx.product(mx.quantize(t), mx.quantize(u)).double().cpu().numpy()
        assert np.array_equal(got[:, :20], want[at]), rows


def test_a_batch_transposed_in_pieces_against_the_definition():
    """60000 inputs, of which 256 rows fit the transposition's workspace: rows of both pieces."""
    import torch
    B = _bcpnn()
    g = np.random.default_rng(4)
    hi, ho, mo, n = 30000, 100, 8, 300
    mask = np.zeros((hi, ho), np.uint8)
    for h in range(ho):
        mask[g.choice(hi, 500 - 3 * h, replace=False), h] = 1
    w = torch.randn(2 * hi, ho * mo, generator=_gen(1), device="cuda")
    b = torch.randn(ho * mo, generator=_gen(2), device="cuda")
    cfg = B.default_config(hi, 2, ho, mo, n, gain=2.0)
    x = torch.rand(n, 2 * hi, generator=_gen(3), device="cuda")
    room = torch.full((2, n + 2, ho * mo), 55.0, device="cuda")
    y, s = room[0, :n], room[1, :n]
    with _mx().Layer(cfg, mask, w, b) as layer:
        layer.forward(x, y, s)
    assert bool((room[:, n:] == 55.0).all())
    rows = [0, 31, 32, 255, 256, 287, 288, 299]
    yo, so, err = mx_plain.forward(cfg, mask, w.cpu().numpy(), b.cpu().numpy(), x[rows].cpu().numpy())
    y, s = y[rows].double().cpu().numpy(), s[rows].double().cpu().numpy()
    assert np.all(np.abs(s - so) <= err)
    rel = np.repeat(mx_plain.softmax_bound(cfg, so, err), mo, 1)
    assert np.all(np.abs(y - yo) <= rel * yo + 2.0 ** -126)


@pytest.mark.parametrize("storage", ["bf16", "m10"])
@pytest.mark.parametrize("pairs", [0, 1])
def test_layer_of_every_storage_format(storage, pairs):
    import torch
    B = _bcpnn()
    cfg = B.default_config(64, 2, 4, 16, 32, alpha=0.05, seed=3, storage=storage, complement_pairs=pairs)
    mask = np.zeros((64, 4), np.uint8)
    for h in range(4):
        mask[h:h + 20 + h, h] = 1
    pixels = torch.rand(32, 64, generator=_gen(1), device="cuda")
    x = torch.stack([pixels, 1 - pixels], 2).reshape(32, 128).contiguous()
    y, s = (torch.empty(32, 64, device="cuda") for _ in range(2))
    with B.Layer(cfg, mask) as trained:
        for _ in range(3):
            trained.train_batch(x)
            trained.structural_update(count=False)
        with _mx().Layer.of(trained) as layer:
            layer.forward(x, y, s)
        st = trained.get_state(("w", "b", "mask"))
    _, so, err = mx_plain.forward(cfg, st["mask"], st["w"], st["b"], x.cpu().numpy())
    assert np.all(np.abs(s.double().cpu().numpy() - so) <= err)
