"""Host threads that call the library at the same time: on one stream, whose
workspace their calls share, and on their own.  Outputs equal those of the same
calls made alone, bit for bit."""
import threading

import pytest

from paper_2607_06763_amd import workloads as W
from tests.attn_ref import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_attn as A
    from paper_2607_06763_amd import gdn_tree as G
    G.lib()
    return A


def run(threads):
    """Each of threads in its own; raises what one raised."""
    errors = []

    def guarded(fn):
        try:
            fn()
        except BaseException as e:
            errors.append(e)
    ts = [threading.Thread(target=guarded, args=(fn,)) for fn in threads]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    if errors:
        raise errors[0]


def calls(A):
    """(call into a tensor, its output alone): attention of a token and of trees, verification above 128 slots."""
    import torch
    from paper_2607_06763_amd import gdn_tree as G
    out = []
    for seed, T, ctx in ((1, 1, [2000, 90]), (2, 40, [700]), (3, 150, [64, 300])):
        c = Case(800 + seed, T, ctx, 8, 2, 128, 64, "bf16", parent=None if T == 1 else "any")
        c.append_slots()
        g, d = c.device(), c.dims()
        out.append((lambda o, s, g=g, d=d: A.attend(d, g["q"], g["kc"], g["vc"], g["table"], g["ctx"], o, meta=g["meta"],
                                                    stream=s), torch.empty_like(g["q"])))
    dt = G.DeviceTree(W.make_random(7400, 2, 200, 1, 2, 64, 64, "bf16", shuffle=True))
    dt.prepare()
    out.append((lambda o, s: dt.verify(out=o, stream=s), torch.empty_like(dt.out)))
    torch.cuda.synchronize()
    for call, want in out:
        call(want, torch.cuda.current_stream())
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("shared", [True, False])
def test_threads(A, shared):
    import torch
    made = calls(A)
    one = torch.cuda.Stream()
    outs = [[torch.full_like(want, float("nan")) for _ in range(25)] for _, want in made]
    streams = [one if shared else torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()

    def loop(n):
        for o in outs[n]:
            made[n][0](o, streams[n])
    print(f"[gpu] {len(made)} threads, one stream: {shared}", flush=True)
    run([lambda n=n: loop(n) for n in range(len(made))])
    torch.cuda.synchronize()
    for (_, want), got in zip(made, outs):
        bits = torch.int16 if want.element_size() == 2 else torch.int32
        assert all(torch.equal(o.view(bits), want.view(bits)) for o in got)
