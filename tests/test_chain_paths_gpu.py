"""gdn_chain on the paths that small batches do not take: every form of the scan,
several passes over the workspace, tensors beyond 2^31 elements, lengths that are
not valid, graphs, streams, threads.  Tolerances: tests/test_chain_gpu.py."""
import threading

import numpy as np
import pytest

from tests.chain_ref import Chain
from tests.guard import check_guards, guarded
from tests.test_chain_gpu import TOL, check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_layer as L
    return L


def ragged(seed, B, T):
    n = np.random.default_rng(seed).integers(0, T + 1, B)
    n[B // 2] = T
    return n.tolist()


# heads times slices of 16 channels: up to 256, up to 512 (two waves a slice), above (one)
FORMS = [
    (3, 2, 6, 128, 64, 150, "bf16", "f32"), (5, 2, 8, 32, 128, 90, "f32", "bf16"), (7, 2, 8, 128, 128, 140, "bf16", "bf16"),
    (9, 4, 16, 64, 64, 130, "f32", "f32"), (12, 4, 16, 32, 64, 100, "bf16", "f32"), (6, 8, 16, 128, 128, 129, "f32", "f32"),
    (12, 4, 16, 16, 128, 130, "bf16", "f32"), (12, 8, 16, 128, 128, 70, "f32", "bf16"), (13, 16, 16, 64, 128, 66, "bf16", "bf16"),
    (40, 2, 16, 16, 16, 65, "f32", "f32"), (33, 2, 8, 32, 32, 70, "bf16", "f32"), (40, 4, 8, 128, 32, 66, "f32", "bf16"),
    (35, 8, 8, 64, 32, 129, "bf16", "bf16"),
]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: ".".join(map(str, f)))
def test_forms_of_the_scan(L, form):
    B, Hk, Hv, dk, dv, T, dt, out = form
    run(L, Chain(500 + B + dv, ragged(B + dk, B, T), Hk, Hv, dk, dv, dt, out, packed=B % 2 == 1, T=T))


@pytest.mark.parametrize("B,T,packed", [(2, 1280, False), (40, 90, True), (1, 3000, False)])
def test_passes_over_the_workspace(L, B, T, packed):
    """64 key heads of 128: a chunk takes 8 MB of it, 33 chunks all."""
    n = ragged(B, B, T) if B > 1 else [T]
    run(L, Chain(600 + B, n, 64, 64, 128, 16, "bf16", packed=packed, T=T))


@pytest.mark.parametrize("n", [5, 100])
def test_rows_beyond_32_bits(L, n):
    """The last tokens of tensors of more than 2^31 values (and 2^32 bytes), rows of 256 heads."""
    import torch
    c = Chain(610, [n], 1, 256, 16, 128, "bf16", "bf16", packed=True, spare=0)
    a = c.device()
    rows = 66000
    assert rows * 256 * 128 > 2 ** 31
    first = rows - n
    big = {}
    for k in ("q", "k", "v", "alpha", "beta", "out"):
        big[k] = torch.empty((rows, *a[k].shape[1:]), dtype=a[k].dtype, device="cuda")
        big[k][first:] = a[k]
    start = torch.tensor([first, rows], dtype=torch.int32, device="cuda")
    d = L.make_chain_dims(1, n, 1, 256, 16, 128, in_dtype="bf16", out_dtype="bf16", rows=rows)
    a2 = dict(a, **big, start=start)
    print(f"[gpu] chain: rows {first} .. {rows} of 256 heads", flush=True)
    L.chain(d, **a2)
    a["out"], = (big["out"][first:].clone(),)
    check(c, a)


@pytest.mark.parametrize("T", [6, 130])
def test_lengths_that_are_not_valid(L, T):
    """They are reported, the sequence keeps its state; the others are as ever."""
    import torch
    for packed in (False, True):
        n = [T, T - 3, T - 1, 2]
        c = Chain(620 + T, n, 1, 2, 32, 32, packed=packed, T=T)
        a = c.device()
        if packed:
            s = a["start"].tolist()
            bad = [([s[0], s[1], s[1] - 1, s[3], s[4]], [1, 2]), ([s[0], s[1], s[2], s[3], c.rows + 1], [3]), ([-1, s[1], s[2], s[3], s[4]], [0]),
                   ([0, s[1], s[2], s[3], -2 ** 31], [3]), ([0, s[1], s[2], s[3], 2 ** 31 - 1], [3])]
        else:
            bad = [([T + 1, n[1], n[2], n[3]], [0]), ([n[0], -1, n[2], n[3]], [1]), ([2 ** 31 - 1, -2 ** 31, n[2], n[3]], [0, 1])]
        for lengths, which in bad:
            a = c.device()
            a["start" if packed else "n_new"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
            print(f"[gpu] chain T={T} packed={packed} lengths {lengths}", flush=True)
            L.chain(c.dims(), **a)
            torch.cuda.synchronize()
            st = a["status"].tolist()
            assert [b for b in range(4) if st[b]] == which and all(st[b] in (0, 9) for b in range(4)), st
            out, S, conv = c.ref()
            for b in range(4):
                got = a["S"][b].double().cpu().numpy()
                if b in which:
                    assert np.array_equal(got, c.S[b].astype(np.float64))
                    assert np.array_equal(a["conv_state_out"][b].cpu().numpy(), c.conv_state[b])
                elif not packed or (lengths[b], lengths[b + 1]) == (c.first[b], c.first[b] + n[b]):
                    assert np.sqrt(((got - S[b]) ** 2).sum()) <= TOL * np.sqrt((S[b] ** 2).sum()), b


def test_nothing_outside_is_written(L):
    import torch
    for n, Hk, Hv, dk, dv, T in (([3, 1], 1, 3, 16, 16, 4), ([70, 0, 130], 2, 2, 32, 16, 131), ([129], 2, 8, 128, 128, 129),
                                 ([65] * 6, 2, 16, 64, 128, 65)):
        c = Chain(630, n, Hk, Hv, dk, dv, T=T)
        a = c.device()
        fulls = {}
        for k in ("S", "out", "conv_state_out"):
            a[k], fulls[k] = guarded(tuple(a[k].shape), fill=a[k])
        L.chain(c.dims(), **a)
        torch.cuda.synchronize()
        for k, f in fulls.items():
            check_guards(f, k)
        check(c, a)


def test_same_inputs_same_bits(L):
    import torch
    for n, T in (([9, 5], 9), ([200, 131], 200)):
        c = Chain(640, n, 2, 4, 64, 64, "bf16", T=T)
        got = []
        for _ in range(3):
            a = c.device()
            L.chain(c.dims(), **a)
            got.append([a[k].clone() for k in ("out", "S", "conv_state_out")])
        for g in got[1:]:
            assert all(torch.equal(x, y) for x, y in zip(g, got[0]))


@pytest.mark.parametrize("n", [[7, 3], [150, 90]])
def test_graph(L, n):
    """Replayed with the program's own work between; every replay against the eager result."""
    import torch
    c = Chain(650, n, 2, 4, 64, 64, "bf16", T=max(n))
    a = c.device()
    s0 = a["S"].clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        L.chain(c.dims(), **a)
    torch.cuda.synchronize()
    want = [a[k].clone() for k in ("out", "S", "conv_state_out")]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        a["S"].copy_(s0)
        L.chain(c.dims(), **a)
    for k in range(4):
        a["out"].fill_(float(k))
        a["conv_state_out"].fill_(3.0)
        if k % 2:  # the same call and others, eager, on the capture stream, which ends before the replay
            with torch.cuda.stream(stream):
                L.chain(c.dims(), **dict(c.device()))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        rows = torch.from_numpy(c.live).cuda()
        x, y = (t.reshape(c.rows, -1)[rows] for t in (a["out"], want[0]))
        assert torch.equal(x, y) and torch.equal(a["S"], want[1]) and torch.equal(a["conv_state_out"], want[2]), k


def test_capture_needs_the_workspace(L):
    """On a stream that has none a capture of the chunked form is refused; of few tokens it is not."""
    import torch
    c = Chain(660, [100], 1, 1, 32, 32)
    few = Chain(661, [3], 1, 1, 32, 32)
    a, b = c.device(), few.device()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    from paper_2607_06763_amd import gdn_tree as G
    with torch.cuda.graph(g, stream=stream):
        with pytest.raises(G.GdnError) as e:
            L.chain(c.dims(), **a)
        L.chain(few.dims(), **b)
    assert e.value.code == G.GDN_EUNSUPPORTED and "captured" in str(e.value)
    g.replay()
    torch.cuda.synchronize()
    check(few, b)


def test_streams_and_threads(L):
    """Calls on streams of their own at once, from two threads each; each stream has its workspace."""
    import torch
    cases = [Chain(670 + i, [130 + 10 * i, 64], 2, 4, 64, 32, "bf16") for i in range(4)]
    args = [[c.device() for _ in range(3)] for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            with torch.cuda.stream(streams[i % 2]):
                for a in args[i]:
                    L.chain(cases[i].dims(), **a)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for c, many in zip(cases, args):
        for a in many:
            check(c, a)


def test_empty(L):
    """No sequence; sequences of no tokens; tensors without rows."""
    import torch
    d = L.make_chain_dims(0, 5, 1, 2, 16, 16, in_dtype="f32")
    z = lambda *s: torch.zeros(*s, device="cuda")
    L.chain(d, z(0, 5, 1, 16), z(0, 5, 1, 16), z(0, 5, 2, 16), z(0, 5, 2), z(0, 5, 2), z(64, 4), z(0, 3, 64), z(0, 3, 64), z(0, 2, 16, 16),
            z(0, 5, 2, 16))
    for T in (0, 4, 40):
        for packed in (False, True):
            c = Chain(680, [0, 0], 1, 2, 16, 16, packed=packed, T=T, spare=0)
            a = c.device()
            L.chain(c.dims(), **a)
            check(c, a)


def test_binding_refuses(L):
    import torch
    c = Chain(690, [4, 4], 1, 2, 16, 16)
    a = c.device()
    for k, v in (("q", a["q"].half()), ("q", a["q"][:, :3]), ("k", a["k"].transpose(1, 2)), ("S", a["S"].cpu()), ("v", None),
                 ("start", torch.zeros(3, dtype=torch.int32, device="cuda")), ("n_new", torch.zeros(2, dtype=torch.int64, device="cuda")),
                 ("out", a["out"].bfloat16())):
        with pytest.raises((ValueError, TypeError)):
            L.chain(c.dims(), **dict(a, **{k: v}))
    x = torch.zeros(4, 2, 8, device="cuda")
    for bad in (dict(gate=x.half()), dict(gate=x[:3]), dict(out=x.transpose(0, 1)), dict(weight=x[0, 0].bfloat16()), dict(weight=x[0, 0, :4]),
                dict(x=x.expand(4, 2, 8)[:, :, ::2]), dict(gate=x[:1].expand(4, 2, 8))):
        with pytest.raises(ValueError):
            L.gate_norm(**dict(dict(x=x, gate=torch.zeros_like(x), out=torch.empty_like(x)), **bad))
    y = torch.zeros(4, 8, device="cuda")
    for bad in (dict(residual=y.bfloat16(), res_out=torch.empty_like(y)), dict(out=y.t()), dict(scale=y[0, :4]), dict(x=y[:, :4])):
        with pytest.raises(ValueError):
            L.add_norm(**dict(dict(x=y, residual=y.clone(), res_out=torch.empty_like(y), out=torch.empty_like(y)), **bad))
