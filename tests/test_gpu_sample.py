"""Tokens drawn from logits on the GPU against a plain 64-bit form: every token, and its log-probability."""
import decimal

import pytest
import torch

import paper_2309_01507_amd as lpmm
import sample_util as ref
from conftest import progress

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


def logits(t, v, dtype, seed, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(t, v, generator=g)).to(dtype), torch.rand(t, generator=g)


def run(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, what="", on_gpu=None, unsure=0):
    on = lambda o: o.to(DEV) if torch.is_tensor(o) else o
    zd = z.to(DEV) if on_gpu is None else on_gpu
    tokens, logprob = lpmm.lpmm_sample(zd, u.to(DEV), on(temperature), on(top_k), on(top_p), on(min_p))
    ref.check(z, u, temperature, top_k, top_p, min_p, tokens, logprob, what, unsure)
    return tokens, logprob


OPTIONS = [{}, {"top_k": 7}, {"top_p": 0.8}, {"min_p": 0.05}, {"temperature": 0.5, "top_k": 40, "top_p": 0.9, "min_p": 0.01},
           {"temperature": 1.7, "top_p": 0.999}, {"top_k": 1}, {"top_p": 0.0}, {"min_p": 1.0}, {"min_p": 2.0}, {"temperature": 0.0, "top_k": 3}]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [1, 2, 63, 64, 65, 255, 257, 1000, 1024, 1025, 4099])
def test_sizes_and_options(v, dtype):
    for n, options in enumerate(OPTIONS):
        z, u = logits(9, v, dtype, 100 * v + n)
        run(z, u, what=f"{v} {options}", **options)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v", [(3, 32000), (2, 50257), (2, 131073), (1, 300001)])
def test_large_vocabularies(t, v, dtype):
    for n, options in enumerate(OPTIONS[:6] + [{"top_k": 2000, "top_p": 0.99}, {"temperature": 4.0, "top_k": v - 1, "top_p": 0.5}]):
        progress(f"sample {t} x {v} {options}")
        z, u = logits(t, v, dtype, v + n)
        z[:, v - v // 50:] = -INF
        run(z, u, what=f"{v} {options}", **options)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [100, 3000, 50257])
def test_equal_logits(v, dtype):
    """Few values: borders fall among equal logits, which the index orders; more of them than a list holds."""
    for n, values in enumerate((1, 2, 5)):
        g = torch.Generator().manual_seed(v + n)
        z = torch.randint(0, values, (6, v), generator=g).to(dtype) - 3
        u = torch.rand(6, generator=g)
        # numbers of equal weights that a rounded share does not hit: kept ones are counted without a doubt
        for options in ({}, {"top_k": v // 3}, {"top_p": 0.37}, {"top_k": v // 2 + 1, "top_p": 0.71}, {"min_p": 0.3, "top_p": 0.55}):
            run(z, u, what=f"{values} values {options}", **options)


def test_each_row_its_own():
    t, v = 200, 2111
    z, u = logits(t, v, F32, 5)
    g = torch.Generator().manual_seed(6)
    heat = 0.2 + 2 * torch.rand(t, generator=g)
    heat[::7] = 0.0
    k = torch.randint(0, 60, (t,), generator=g, dtype=torch.int32)
    k[::5] = v + 3
    p, least = torch.rand(t, generator=g), 0.2 * torch.rand(t, generator=g)
    p[::4], least[::3] = 1.0, 0.0
    run(z, u, heat, k, p, least, what="each")
    # values that a call for all rows refuses
    heat[1], heat[2], heat[3], heat[4] = -1.0, NAN, INF, 1e-30
    k[5], k[6], p[8], p[9], p[10], least[11], least[12] = -4, -2 ** 31, NAN, -3.0, INF, NAN, -1.0
    tokens, logprob = lpmm.lpmm_sample(z.to(DEV), u.to(DEV), heat.to(DEV), k.to(DEV), p.to(DEV), least.to(DEV))
    heat[1] = heat[2] = 0.0
    heat[3] = 1e30                                            # all weights 1, to 30 digits
    k[5] = k[6] = 0
    p[8], p[9], least[11], least[12] = 1.0, 0.0, 0.0, 0.0
    ref.check(z, u, heat, k, p, least, tokens, logprob, "odd values")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_and_unusual_rows(dtype):
    v = 1500
    low = torch.finfo(dtype).min
    z, u = logits(12, v, dtype, 8)
    z[0] = -INF
    z[1] = low
    z[2, 5:] = -INF
    z[3, :-1] = -INF
    z[4, 700] = NAN
    z[5, 3] = z[5, 900] = INF
    z[6, 3], z[6, 9] = INF, -INF
    z[7] = INF
    z[8, ::2] = low
    z[9] = -INF
    z[9, 44] = NAN
    z[10, 0], z[10, 1] = torch.finfo(dtype).max, low
    z[11] = 0.0
    z[11, ::3] = -0.0
    for options in ({}, {"top_k": 4}, {"top_p": 0.6}, {"top_k": 900, "top_p": 0.95}, {"min_p": 0.5}, {"temperature": 0.0}, {"temperature": 0.01, "top_p": 0.9}):
        run(z, u, what=f"{options}", **options)


def test_numbers_at_the_ends():
    """u of 0, just below 1, 1, negative, NaN: the first kept, the last kept."""
    v = 333
    z, _ = logits(7, v, F32, 9)
    z[:] = z[0]
    z[:, 0] = z[:, -1] = -INF
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, NAN, INF, -INF])
    for options in ({}, {"top_k": 11}):
        tokens, _ = lpmm.lpmm_sample(z.to(DEV), u.to(DEV), **options)
        kept = torch.topk(z[0], options.get("top_k", v - 2)).indices
        first, last = int(kept.min()), int(kept.max())
        assert tokens.tolist() == [first, last, last, first, first, last, first]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_anywhere(dtype):
    """Rows apart, off every boundary, and beyond 2^31 elements"""
    z, u = logits(5, 777, dtype, 10)
    for gap, off in ((1, 1), (3, 5), (0, 3)):
        room = torch.full((5 * (777 + gap) + off,), NAN, dtype=dtype, device=DEV)
        view = room[off:].view(5, 777 + gap)[:, :777]
        view.copy_(z)
        run(z, u, top_p=0.9, what=f"{gap} {off}", on_gpu=view)
    far = torch.empty(2 ** 31 + 1000, dtype=dtype, device=DEV)
    view = far.as_strided((2, 777), (2 ** 31 + 64, 1))
    view.copy_(z[:2])
    run(z[:2], u[:2], top_k=30, what="far", on_gpu=view)


def test_no_rows_and_given_outputs():
    z = torch.zeros(0, 100, device=DEV)
    tokens, logprob = lpmm.lpmm_sample(z, torch.zeros(0, device=DEV))
    assert tokens.shape == logprob.shape == (0,) and tokens.dtype == torch.int64
    z, u = logits(4, 900, F32, 11)
    z, u = z.to(DEV), u.to(DEV)
    want = lpmm.lpmm_sample(z, u, top_p=0.9)
    room, lp = torch.full((6,), 77, device=DEV), torch.full((6,), 7.0, device=DEV)
    got = lpmm.lpmm_sample(z, u, top_p=0.9, tokens=room[1:5], logprob=lp[1:5])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert room[[0, 5]].tolist() == [77, 77] and lp[[0, 5]].tolist() == [7.0, 7.0]


@pytest.mark.parametrize("t,v", [(20, 9001), (20, 34817)])
def test_on_a_stream_and_captured(t, v):
    """The same bits on another stream and from a captured graph, replayed with other logits and numbers in between; a row's one workgroup, and several"""
    z, u = logits(t, v, BF16, 12)
    z, u = z.to(DEV), u.to(DEV)
    sets = [(z.clone(), u.clone()), (z.flip(0).contiguous(), u.flip(0).contiguous()), (z * 0.5, 1 - u)]
    options = dict(temperature=0.9, top_k=500, top_p=0.95, min_p=0.001)
    want = [lpmm.lpmm_sample(a, b, **options) for a, b in sets]
    tokens, logprob = torch.empty(t, dtype=torch.int64, device=DEV), torch.empty(t, device=DEV)
    room = torch.empty(lpmm.lib().lpmm_sample_workspace_bytes(t, v), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lpmm.lpmm_sample(z, u, **options, tokens=tokens, logprob=logprob, workspace=room, stream=s)
    s.synchronize()
    assert torch.equal(tokens, want[0][0]) and torch.equal(logprob, want[0][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lpmm.lpmm_sample(z, u, **options, tokens=tokens, logprob=logprob)
    for n in (0, 1, 2, 1, 0):
        z.copy_(sets[n][0])
        u.copy_(sets[n][1])
        graph.replay()
        assert torch.equal(tokens, want[n][0]) and torch.equal(logprob, want[n][1])
        torch.randn(1000, device=DEV).sum().item()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v", [(1, 25087), (1, 25088), (3, 26201), (5, 27136), (17, 33301), (64, 57344), (65, 57900), (1, 524288), (1, 524289)])
def test_few_rows(t, v, dtype):
    """Rows shared by several workgroups, and sizes next to where that begins and ends; the list's way and the lines' way"""
    for n, options in enumerate(OPTIONS + [{"top_k": 900, "top_p": 0.9}, {"top_k": 1500}, {"temperature": 3.0, "top_p": 0.6, "min_p": 0.1}]):
        if t > 60 and n % 3:
            continue
        z, u = logits(t, v, dtype, 7 * v + t + n)
        run(z, u, what=f"{t} x {v} {options}", **options)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_few_rows_of_equal_and_unusual_logits(dtype):
    v = 31000
    low = torch.finfo(dtype).min
    for n, options in enumerate(({}, {"top_k": 4}, {"top_k": 3000}, {"top_p": 0.6}, {"top_k": 700, "top_p": 0.95, "min_p": 0.001}, {"min_p": 0.5, "top_p": 0.7}, {"min_p": 1.0},
                                 {"min_p": 1.5, "top_p": 0.3}, {"temperature": 0.0}, {"temperature": 0.01, "top_p": 0.9})):
        z, u = logits(12, v, dtype, 60 + n)
        z[0] = -INF
        z[1] = low
        z[2, 5:] = -INF
        z[3, :-1] = -INF
        z[4, 17000] = NAN
        z[5, 3] = z[5, 30900] = INF
        z[6, 3], z[6, 9] = INF, -INF
        z[7] = INF
        z[8, ::2] = low
        z[9] = (z[9] * 2).round()
        z[10] = 0.25
        z[11] = z[11].round()
        run(z, u, what=f"{options}", **options)


def test_workspaces():
    """A call on a stream of its own is given one; two calls at once have one each; one that is too small, off its boundary or missing is refused"""
    z, u = logits(2, 26000, F32, 70)
    z, u = z.to(DEV), u.to(DEV)
    need = lpmm.lib().lpmm_sample_workspace_bytes(2, 26000)
    assert need > 0 and lpmm.lib().lpmm_sample_workspace_bytes(65, 90000) == lpmm.lib().lpmm_sample_workspace_bytes(2, 25599) == 0
    want = lpmm.lpmm_sample(z, u, top_p=0.9)
    room = [torch.randint(0, 256, (need,), dtype=torch.uint8, device=DEV) for _ in range(2)]
    out = [(torch.empty(2, dtype=torch.int64, device=DEV), torch.empty(2, device=DEV)) for _ in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, r, o in zip(streams, room, out):
            lpmm.lpmm_sample(z, u, top_p=0.9, tokens=o[0], logprob=o[1], workspace=r, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], want[0]) and torch.equal(o[1], want[1]) for o in out)
    for bad in (room[0][:-1], room[0][1:]):
        with pytest.raises(lpmm.LpmmError):
            lpmm.lpmm_sample(z, u, workspace=bad)
    with pytest.raises(ValueError):
        lpmm.lpmm_sample(z, u, tokens=out[0][0], logprob=out[0][1], stream=streams[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [130, 2500, 9000, 21000])
def test_borders_of_shares(v, dtype):
    """The share's border next to the least probability's, in the first and the last range of logits, among equal ones, and logits that sit on the ranges' own borders.  Shares of
    1 - 2^-20 and more end among weights that are near 2^-46: of 70 rows up to four end too near to one to say which."""
    for n, spread in enumerate((0.001, 0.3, 3.0, 40.0)):
        z, u = logits(70, v, dtype, v + n, spread)
        z[20:40] = (z[20:40] * (512 / 7)).round() * (7 / 512)            # 28 / 2048: the width of a range at temperature 1
        z[40:60] = (z[40:60] * 2).round() / 2
        z[60:, ::3] = -INF
        p = torch.tensor([0.0, 1e-30, 0.01, 0.5, 0.9, 0.999, 1 - 2**-20, 1 - 2**-24, 0.7, 0.95]).repeat(7)
        least = torch.tensor([0.0, 0.0, 0.001, 0.1, 0.5, 0.9, 0.999]).repeat_interleave(10)
        run(z, u, 1.0, 0, p, least, what=f"{v} {spread}", unsure=4)
        run(z, u, torch.linspace(0.05, 4, 70), 0, p, least[torch.arange(70) * 7 % 70], what=f"{v} {spread}, temperatures", unsure=4)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v", [(6, 3000), (6, 27700)])
def test_extreme_temperatures(t, v, dtype):
    """Where 1 / temperature, differences or their products leave fp32's range; logits at its ends"""
    for n, heat in enumerate((2.0**-149, 2.0**-126, 1e-30, 1e30, 3e38, INF)):
        z, u = logits(t, v, dtype, 500 + n)
        z[1] = z[1] * 1e-38
        z[2] = torch.where(z[2] > 0, z[2] * 1e37, z[2])
        z[3, 5], z[3, 9] = torch.finfo(dtype).max, torch.finfo(dtype).min
        z[4, ::2] = -INF
        z[5, 7] = z[5, 70] = INF
        for options in ({}, {"top_p": 0.7}, {"top_p": 0.9, "min_p": 0.3}, {"top_k": 50, "top_p": 0.9}):
            run(z, u, temperature=heat, what=f"{heat} {options}", **options)


@pytest.mark.parametrize("t,v", [(3, 900), (2, 26000)])
def test_rows_far_apart(t, v):
    """Rows that begin beyond 2^32 bytes"""
    z, u = logits(t, v, BF16, 80 + v)
    room = torch.empty(2**31 + v, dtype=BF16, device=DEV)
    far = room.as_strided((t, v), (2**31 // (t - 1), 1))
    far.copy_(z)
    for options in ({"top_p": 0.9}, {"top_k": 20, "min_p": 0.01}):
        run(z, u, what=f"{v} {options}", on_gpu=far, **options)


def test_many_rows():
    """More rows than a launch's second dimension could hold, each like that of a small call"""
    z, u = logits(7, 33, F32, 90)
    want = run(z, u, top_p=0.8, what="small")
    many = 10001
    tokens, logprob = lpmm.lpmm_sample(z.to(DEV).repeat(many, 1), u.to(DEV).repeat(many), top_p=0.8)
    assert torch.equal(tokens, want[0].repeat(many)) and torch.equal(logprob, want[1].repeat(many))


def test_one_workspace_for_two_graphs():
    """Replayed one after the other, as calls on one stream"""
    sets = [logits(3, 26200, F32, 91), logits(5, 30001, BF16, 92)]
    sets = [(z.to(DEV), u.to(DEV)) for z, u in sets]
    want = [lpmm.lpmm_sample(z, u, top_k=30, top_p=0.9) for z, u in sets]
    room = torch.empty(max(lpmm.lib().lpmm_sample_workspace_bytes(*z.shape) for z, _ in sets), dtype=torch.uint8, device=DEV)
    outs = [(torch.empty(z.shape[0], dtype=torch.int64, device=DEV), torch.empty(z.shape[0], device=DEV)) for z, _ in sets]
    graphs = []
    for (z, u), o in zip(sets, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            lpmm.lpmm_sample(z, u, top_k=30, top_p=0.9, tokens=o[0], logprob=o[1], workspace=room)
    for _ in range(3):
        for g, o in zip(graphs, outs):
            o[0].zero_()
            g.replay()
        room.fill_(255)
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v", [(8, 700), (8, 3000), (8, 29000), (1, 24577 + 511)])
def test_infinite_logits_at_any_temperature(t, v, dtype):
    """Only they are drawn, whatever min_p says alone, with top_k and with top_p; in lists, by lines, and where several workgroups share a row"""
    for n, heat in enumerate((1.0, 3e38, INF)):
        z, u = logits(t, v, dtype, 900 + n)
        z[0, 3] = z[0, 41] = z[0, v - 1] = INF
        if t > 1:
            z[1, ::2] = INF
            z[2] = INF
            z[3, 77], z[3, ::3] = INF, -INF
            z[4, -1] = INF
        for options in ({"min_p": 0.3}, {"min_p": 1e-30}, {"min_p": 0.999, "top_p": 0.6}, {"min_p": 0.5, "top_k": 2}, {"min_p": 0.5, "top_k": 600}, {"min_p": 0.1, "top_k": 50, "top_p": 0.7},
                        {"min_p": 1.0}, {"min_p": 1.0, "top_k": 5}):
            progress(f"sample {t} x {v} {heat} {options}")
            if options["min_p"] == 1.0 and heat < INF:
                # exp(x) is below 1 for every x below 0, where 64 bits round it to 1 for those near 0: what is kept of the first top_k are those that equal the largest, with weights of 1
                same = torch.where(z == z.amax(1, keepdim=True), z, torch.full_like(z, -INF))
                got = lpmm.lpmm_sample(z.to(DEV), u.to(DEV), heat, **options)
                ref.check(same, u, heat, options.get("top_k", 0), 1.0, 0.0, *got, f"{heat} {options}")
            else:
                run(z, u, temperature=heat, what=f"{heat} {options}", **options)


# N logits whose weight w has its binary logarithm next to -1/2, where a series for powers of two is farthest from them, and M of weight 1.  u: the sum of the N comes just before u times
# that of all.  p: of them all, largest first, p leaves the M and a tenth of the N, whose sum just reaches p times that of all.
NEAR = [("u", F32, 608, 397, "-0x1.62c51ep-2", "1", "0x1.0a34f6p-1"), ("u", F32, 15063, 14528, "-0x1.6270fcp-2", "1", "0x1.b146e0p-2"),
        ("u", F32, 13792, 15699, "-0x1.62c69ap-2", "1", "0x1.8866bep-2"), ("u", BF16, 807, 805, "-1", "0x1.71a71ap+1", "0x1.a8d8bap-2"),
        ("u", BF16, 665, 811, "-1", "0x1.718dacp+1", "0x1.77dee6p-2"), ("u", BF16, 475, 312, "-1", "0x1.71b0acp+1", "0x1.097a34p-1"),
        ("p", F32, 14785, 15177, "-0x1.62a798p-2", "1", "0x1.440446p-1"), ("p", F32, 15406, 14305, "-0x1.62b674p-2", "1", "0x1.38c32ep-1"),
        ("p", F32, 13495, 15529, "-0x1.626bb8p-2", "1", "0x1.508ee4p-1"), ("p", F32, 783, 714, "-0x1.628a4cp-2", "1", "0x1.369ddcp-1"),
        ("p", F32, 300, 362, "-0x1.62723ap-2", "1", "0x1.55b210p-1")]


@pytest.mark.parametrize("what,dtype,low,high,z,heat,number", NEAR)
def test_weights_whose_errors_add_up(what, dtype, low, high, z, heat, number):
    """Each weight may be off by 2^-47 and a little, all of them in the same direction: a border may move by (low + high) 2^-47, and is at least four times that away."""
    z, heat, number = (float.fromhex(x) if "0x" in x else float(x) for x in (z, heat, number))
    with decimal.localcontext() as exact:
        exact.prec = 50
        w = (decimal.Decimal(z) / decimal.Decimal(heat)).exp()
        ahead = low * w if what == "u" else high + low // 10 * w
        off = decimal.Decimal(number) * (high + low * w) - ahead
    v = low + high
    assert 4 * v * 2.0 ** -47 < (off if what == "u" else -off) < v * 2.0 ** -43
    parts = [torch.full((low,), z), torch.zeros(high)]
    row = torch.cat(parts if what == "u" else parts[::-1])
    last = 1 - 2.0 ** -24                                       # draws the last one that is kept: the sum of thousands of weights lacks less than one of them
    token = low if what == "u" else high + low // 10 - 1
    for t in (1, 66):                                           # long rows by several workgroups, or one
        for listed in ((False, True) if v < 1024 else (False,)):
            logits = torch.cat([row, torch.full((1,), -INF)]).to(dtype).repeat(t, 1).to(DEV)
            u = torch.full((t,), number if what == "u" else last, device=DEV)
            tokens, _ = lpmm.lpmm_sample(logits, u, heat, v if listed else 0, 1.0 if what == "u" else number)
            assert tokens.tolist() == [token] * t, f"{t} rows, {listed}"
