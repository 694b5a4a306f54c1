"""Every way of a product of 8-bit matrices: the tiles that the planner chooses between, their
last rounds in sub-tiles, K slices and their join, blocks straight from memory; in replayed
graphs, on other streams, and beyond what 32-bit offsets reach."""
import pytest
import torch

import qint_reference as ref
from paper_2606_29094_amd import dlm
from test_gpu_qint import BF16, F32, _check_linear, _empty, _matrix, _randn

pytestmark = pytest.mark.gpu
DIRECT = -1
STORE, ADD, SWIGLU = dlm.DLM_QINT_STORE, dlm.DLM_QINT_ADD, dlm.DLM_QINT_SWIGLU


# (rows, n, k, epilogue) and what the planner takes on 256 CUs: configuration, K slices, sub-tiles
WAYS = [
    (1, 2, 1, STORE, (DIRECT, 1, 0)), (1, 2, 1, ADD, (DIRECT, 1, 0)), (1, 2, 1, SWIGLU, (DIRECT, 1, 0)),
    (1, 4, 14430, SWIGLU, (DIRECT, 8, 0)), (1, 4, 14735, ADD, (DIRECT, 8, 0)),
    (1, 4, 14797, STORE, (DIRECT, 8, 0)), (383, 24812, 1, SWIGLU, (6, 1, 0)),
    (354, 30204, 1, STORE, (6, 1, 0)), (395, 32220, 1, ADD, (6, 1, 0)), (645, 24830, 1, STORE, (6, 1, 4)),
    (3224, 922, 14149, ADD, (6, 4, 0)), (195, 35842, 1, SWIGLU, (21, 1, 0)),
    (227, 34644, 1, STORE, (21, 1, 0)), (604, 14650, 1, ADD, (21, 1, 0)), (985, 16782, 2, ADD, (21, 1, 2)),
    (4102, 146, 4620, STORE, (21, 4, 2)), (2060, 162, 8934, ADD, (21, 8, 2)),
    (4677, 168, 4029, SWIGLU, (21, 4, 2)), (1025, 2, 1, STORE, (22, 1, 0)), (1031, 2, 1, ADD, (22, 1, 0)),
    (1063, 2, 1, SWIGLU, (22, 1, 0)), (645, 2, 1, SWIGLU, (29, 1, 4)), (582, 2578, 1, STORE, (29, 1, 4)),
    (835, 1832, 1, ADD, (29, 1, 4)), (837, 2140, 1, SWIGLU, (29, 1, 2)),
    (197, 22092, 1, STORE, (29, 1, 0)), (646, 2, 2123, SWIGLU, (29, 2, 4)),
    (656, 2, 4193, ADD, (29, 4, 4)), (681, 2, 3983, STORE, (29, 4, 4)),
    (4255, 2, 4000, SWIGLU, (29, 4, 2)), (4142, 4, 8090, ADD, (29, 8, 0)),
    (2727, 644, 1922, SWIGLU, (42, 1, 2)), (1197, 1644, 1938, ADD, (42, 1, 2)),
    (1289, 1574, 1922, STORE, (42, 1, 2)), (1218, 148, 8221, ADD, (42, 8, 2)),
    (1164, 156, 8492, STORE, (42, 8, 2)), (1242, 154, 8644, SWIGLU, (42, 8, 2)),
    (591, 16488, 1, ADD, (70, 1, 0)), (417, 24662, 1, STORE, (70, 1, 0)),
    (4340, 216, 18224, ADD, (70, 8, 0)), (17, 2, 1, SWIGLU, (80, 1, 0)),
    (165, 4266, 135, STORE, (80, 1, 0)), (141, 5274, 144, ADD, (80, 1, 0)),
    (17, 2, 2469, SWIGLU, (80, 2, 0)), (17, 2, 3071, STORE, (80, 2, 0)), (18, 2, 3206, ADD, (80, 2, 0)),
    (132, 5474, 1, SWIGLU, (81, 1, 0)), (260, 4646, 1, ADD, (81, 1, 0)), (300, 4298, 1, STORE, (81, 1, 0)),
    (76, 2092, 4051, ADD, (81, 4, 0)), (132, 1540, 4091, SWIGLU, (81, 4, 0)),
    (11, 4098, 5119, STORE, (81, 4, 0)), (17, 33958, 1, SWIGLU, (83, 1, 0)),
    (44, 32782, 2, STORE, (83, 1, 0)), (44, 33040, 76, ADD, (83, 1, 0)), (2, 8250, 6122, ADD, (83, 4, 0)),
    (5, 8686, 7125, SWIGLU, (83, 4, 0)), (7, 9902, 7036, STORE, (83, 4, 0)),
    (326, 4206, 1, SWIGLU, (84, 1, 0)), (390, 3988, 1, STORE, (84, 1, 0)), (429, 3708, 1, ADD, (84, 1, 0)),
    (395, 416, 8165, SWIGLU, (84, 8, 0)), (409, 394, 9439, STORE, (84, 8, 0)),
    (138, 2766, 4397, ADD, (84, 4, 0)), (100, 14248, 1, STORE, (85, 1, 0)),
    (104, 13454, 1, SWIGLU, (85, 1, 0)), (97, 14806, 1, ADD, (85, 1, 0)),
    (203, 2188, 4232, SWIGLU, (85, 4, 0)), (205, 2402, 4232, ADD, (85, 4, 0)),
    (208, 2462, 4254, STORE, (85, 4, 0)), (133, 18086, 1, SWIGLU, (86, 1, 0)),
    (129, 19130, 1, ADD, (86, 1, 0)), (77, 33530, 1, STORE, (86, 1, 0)),
    (129, 4598, 9627, STORE, (86, 4, 0)), (527, 1580, 1, SWIGLU, (87, 1, 2)),
    (514, 3268, 1, STORE, (87, 1, 0)), (518, 3752, 1, ADD, (87, 1, 0)),
    (528, 4, 18065, STORE, (87, 16, 2)), (539, 8, 17446, ADD, (87, 16, 2)),
    (637, 2, 19324, SWIGLU, (87, 16, 2)), (623, 782, 4057, SWIGLU, (87, 4, 0)),
    (321, 2, 1, SWIGLU, (88, 1, 4)), (520, 2778, 1, SWIGLU, (88, 1, 2)), (554, 2852, 1, STORE, (88, 1, 2)),
    (618, 3048, 1, ADD, (88, 1, 2)), (516, 5410, 1, ADD, (88, 1, 0)), (325, 2, 2166, SWIGLU, (88, 2, 4)),
    (334, 2, 4028, ADD, (88, 4, 4)), (339, 2, 4206, STORE, (88, 4, 4)),
    (523, 684, 5037, STORE, (88, 4, 2)), (536, 664, 11237, ADD, (88, 8, 0)),
    (781, 4136, 1, SWIGLU, (89, 1, 0)), (794, 4198, 1, ADD, (89, 1, 0)), (386, 9550, 1, STORE, (89, 1, 0)),
    (546, 1624, 4227, STORE, (89, 4, 0)), (642, 1370, 4863, SWIGLU, (89, 4, 0)),
    (751, 1466, 4507, ADD, (89, 4, 0)), (257, 16510, 1, SWIGLU, (90, 1, 0)),
    (254, 16918, 1, STORE, (90, 1, 0)), (104, 37364, 1, ADD, (90, 1, 0)),
    (114, 4110, 15912, STORE, (90, 8, 0)), (853, 4172, 1, STORE, (92, 1, 0)),
    (878, 4268, 1, SWIGLU, (92, 1, 0)), (975, 4458, 1, ADD, (92, 1, 0)),
    (662, 774, 8271, STORE, (92, 8, 0)), (858, 580, 8505, SWIGLU, (92, 8, 0)),
    (818, 582, 8957, ADD, (92, 8, 0)), (332, 18022, 1, STORE, (93, 1, 0)),
    (245, 24290, 1, ADD, (93, 1, 0)), (277, 22242, 1, SWIGLU, (93, 1, 0)),
    (789, 1064, 12201, SWIGLU, (93, 8, 0)), (17, 2, 1, STORE, (94, 1, 0)), (17, 2, 1, ADD, (94, 1, 0)),
    (64, 2048, 2048, STORE, (94, 1, 0)), (128, 4096, 1100, ADD, (94, 1, 0)),
    (70, 689, 1031, STORE, (94, 1, 0)), (33, 4600, 3000, ADD, (94, 1, 0))]


@pytest.mark.parametrize("m,n,k,epilogue,way", WAYS)
def test_way(gpu, m, n, k, epilogue, way):
    assert dlm.debug_qint_linear_plan(m, n, k, epilogue)[:3] == way
    name = {v: k for k, v in dlm.QINT_EPILOGUES.items()}[epilogue]
    for dtype in ((F32,) if epilogue == ADD else (F32, BF16)):
        for pad in (0, 1):
            _check_linear(gpu, m, n, k, name, dtype, pad=pad, seed=m)


@pytest.mark.parametrize("m,n,k", [(8200, 520, 300), (8193, 1030, 140), (12345, 94, 257)])
@pytest.mark.parametrize("epilogue", ["store", "add", "swiglu"])
def test_tiles_in_groups(gpu, m, n, k, epilogue):
    """Row tiles in groups of eight, the last group smaller, whole tiles and sub-tiles."""
    assert dlm.debug_qint_linear_plan(m, n, k, dlm.QINT_EPILOGUES[epilogue])[3] == 8
    _check_linear(gpu, m, n, k, epilogue, F32, seed=m)


def test_ways_are_all_there():
    """Every configuration that the planner takes over a wide range of sizes is tested above."""
    import random
    rng, seen = random.Random(7), set()
    size = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    for _ in range(20000):
        n, k = rng.choice([(4096, 4096), (12288, 4096), (24576, 4096), (4096, 12288), (4608, 3584), (3584, 18944),
                           (37888, 3584), (1376, 256), (2 * size(1, 20000), size(1, 40000))])
        e = rng.choice([STORE, ADD, SWIGLU])
        cfg, slices, sub, _ = dlm.debug_qint_linear_plan(size(1, 8192), n, k, e)
        seen.add((cfg, slices > 1))
    assert seen <= {(w[4][0], w[4][1] > 1) for w in WAYS}


# ------------------------------------------------------------------ graphs
GRAPHS = [(5, 258, 4000, "store", BF16), (7, 30, 30000, "swiglu", F32), (40, 3584, 9000, "add", F32),
          (64, 130, 20000, "swiglu", BF16), (300, 1030, 700, "swiglu", BF16), (1100, 2050, 600, "add", F32)]


@pytest.mark.parametrize("m,n,k,epilogue,dtype", GRAPHS)
def test_replayed_graph(gpu, m, n, k, epilogue, dtype):
    """A layer's run of operators in a graph: each replay, between eager calls on other inputs,
    gives the eager calls' bits."""
    epi = dlm.QINT_EPILOGUES[epilogue]
    w, _, _ = _matrix(gpu, n, k, seed=1)
    cols = n // 2 if epilogue == "swiglu" else n
    h, part, g = torch.empty(m, k, device=gpu), torch.empty(2, m, k, device=gpu), torch.empty(k, device=gpu)
    s, y, r = torch.empty(m, k, device=gpu), torch.empty(m, cols, dtype=dtype, device=gpu), torch.empty(m, cols, device=gpu)
    x, z = _empty(gpu, m, k), _empty(gpu, m, cols)
    out = torch.empty(m, cols, device=gpu)
    ws = torch.empty(max(256, dlm.qint_linear_workspace(m, w, epi)), dtype=torch.uint8, device=gpu)

    def inputs(seed):
        for i, t in enumerate((h, part, g, r)):
            t.copy_(_randn(*t.shape, seed=seed + 10 * i))
        ws.fill_(seed)
        for q in (x, z):
            q._keep[0].fill_(seed)
        y.fill_(seed)

    def call():
        dlm.qint_norm(h, g, 1e-5, x, add=part, h_out=s)
        dlm.qint_linear(x, w, y, epi, ws, residual=r if epilogue == "add" else None)
        dlm.qint_pack(y, z)
        dlm.qint_unpack(z, out)

    result = lambda: [t.clone() for t in (s, y, out, *x._keep, *z._keep)]
    same = lambda a, b: all(torch.equal(p, q) for p, q in zip(a, b))
    want = {}
    for seed in (1, 2, 3):
        inputs(seed)
        call()
        torch.cuda.synchronize()
        want[seed] = result()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (2, 1, 3, 1):
        inputs(seed)
        graph.replay()
        torch.cuda.synchronize()
        assert same(result(), want[seed]), seed
        inputs(3)
        call()                              # an eager call between the replays
        assert same(result(), want[3])


def test_two_streams_at_once(gpu):
    """Calls of every kind on two streams, each with its own buffers, give what they give alone."""
    m, n, k = 60, 3584, 9000
    assert dlm.debug_qint_linear_plan(m, n, k)[1] > 1          # (a workspace each)
    w, _, _ = _matrix(gpu, n, k, seed=1)
    states = []
    for i in range(2):
        states.append(dict(h=_randn(m, k, seed=i).to(gpu), g=_randn(k, seed=9).to(gpu), x=_empty(gpu, m, k),
                           y=torch.empty(m, n, device=gpu), st=torch.cuda.Stream(),
                           ws=torch.empty(dlm.qint_linear_workspace(m, w), dtype=torch.uint8, device=gpu)))

    def call(s, stream=None):
        dlm.qint_norm(s["h"], s["g"], 1e-5, s["x"], stream=stream)
        dlm.qint_linear(s["x"], w, s["y"], workspace=s["ws"], stream=stream)

    want = []
    for s in states:
        call(s)
        torch.cuda.synchronize()
        want.append(s["y"].clone())
        s["y"].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(states):
            if i:
                call(s, s["st"].cuda_stream)          # the stream as an argument
            else:
                with torch.cuda.stream(s["st"]):      # or the current one
                    call(s)
    torch.cuda.synchronize()
    for s, y in zip(states, want):
        assert torch.equal(s["y"], y)


# ------------------------------------------------------------------- large
def test_rows_beyond_32_bit_offsets(gpu):
    """More codes than the tiles' offsets reach (2^33 bytes): the rows are taken in turn."""
    k, m = 131000, 65700
    wide = ref.row_bytes(k)
    assert m * wide > 1 << 33
    codes = torch.zeros(m, wide, dtype=torch.int8, device=gpu)
    at = [0, 1, 40000, 65279, 65280, 65281, 65535, 65536, 65699]
    for i, r in enumerate(at):
        codes[r, :k] = torch.randint(-127, 128, (k,), generator=torch.Generator().manual_seed(i)).to(torch.int8).to(gpu)
    scales = torch.linspace(0.5, 1.5, m, device=gpu)
    x = dlm.make_qint(codes, scales, m, k)
    some = dlm.make_qint(codes[at].contiguous(), scales[at].contiguous(), len(at), k)
    for n, epilogue, dtype in ((6, STORE, F32), (5, ADD, F32), (6, SWIGLU, BF16)):
        w, _, _ = _matrix(gpu, n, k, seed=n)
        cols = n // 2 if epilogue == SWIGLU else n
        r = _randn(m, cols, seed=3).to(gpu) if epilogue == ADD else None
        y, z = torch.empty(m, cols, dtype=dtype, device=gpu), torch.empty(len(at), cols, dtype=dtype, device=gpu)
        ws = torch.empty(max(1, dlm.qint_linear_workspace(m, w, epilogue),
                             dlm.qint_linear_workspace(len(at), w, epilogue)), dtype=torch.uint8, device=gpu)
        dlm.qint_linear(x, w, y, epilogue, ws, residual=r)
        dlm.qint_linear(some, w, z, epilogue, ws, residual=None if r is None else r[at].contiguous())
        assert torch.equal(y[at], z)
        rest = torch.ones(m, dtype=torch.bool)
        rest[at] = False
        assert torch.equal(y[rest], (torch.zeros_like(y) if r is None else r)[rest])


def test_weights_beyond_32_bit_offsets(gpu):
    """A weight matrix of more than 2^32 bytes, and outputs of more than 2^31 elements."""
    n, k = 34000, 131000
    w = dlm.make_qint(torch.zeros(n, ref.row_bytes(k), dtype=torch.int8, device=gpu), torch.ones(n, device=gpu), n, k)
    at = [0, 16999, 17000, 33000, 33999]
    rows = ref.pack(_randn(len(at), k, seed=1))[0]
    w._keep[0][at] = rows.to(gpu)
    for m in (3, 40, 300):
        x, xc, xs = _matrix(gpu, m, k, seed=m)
        for epilogue, cols in ((STORE, n), (SWIGLU, n // 2)):
            y = torch.empty(m, cols, device=gpu)
            ws = torch.empty(max(1, dlm.qint_linear_workspace(m, w, epilogue)), dtype=torch.uint8, device=gpu)
            dlm.qint_linear(x, w, y, epilogue, ws)
            p, bound = ref.product(xc, xs, rows[:, :k], torch.ones(len(at)))
            if epilogue == STORE:
                assert bool(((y[:, at].cpu().double() - p).abs() <= bound).all())
                assert int((y != 0).any(0).sum()) <= len(at)
            else:          # gate 0 with up 17000, 16999 with 33999; 16000's up is 33000, its gate 0
                for col, gate, up in ((0, 0, 2), (16999, 1, 4)):
                    want, b = ref.swiglu(p[:, [gate, up]], bound[:, [gate, up]])
                    assert bool(((y[:, col].cpu().double() - want[:, 0]).abs() <= b[:, 0]).all())
                assert int((y != 0).any(0).sum()) <= 2
    del w
    m, n, k = 40000, 60000, 130                       # 2.4e9 outputs
    x, xc, xs = _matrix(gpu, m, k, seed=1)
    w, wc, ws = _matrix(gpu, n, k, seed=2)
    y = torch.empty(m, n, dtype=BF16, device=gpu)
    dlm.qint_linear(x, w, y)
    rows = torch.tensor([0, 20000, 35790, 35791, 35792, 39999])          # around 2^31 elements
    p, bound = ref.product(xc[rows], xs[rows], wc, ws)
    assert bool(((y[rows.to(gpu)].cpu().double() - p).abs() <= bound + ref.half_ulp(p.abs() + bound, BF16)).all())
