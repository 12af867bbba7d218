"""The operators around the output layer together, as a training step and a served token use them: on another stream behind long work, captured into
graphs that share a workspace and are replayed between eager work."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: the HIP path has no CPU fallback")
    from paper_2409_13313_amd import lm
    return lm


class Step:
    """A training step of a layer, its weights stored in 4 bits, and tokens through them."""
    def __init__(self, lm, m, n, p, kind, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.lm, self.sizes = lm, (m, n, p)
        self.new = {"X": torch.randn((m, n), device="cuda", generator=gen).to(kind), "W": (torch.randn((p, n), device="cuda", generator=gen) * 0.05).to(kind),
                    "y": torch.randint(0, p, (m,), device="cuda", generator=gen), "g": torch.rand(m, device="cuda", generator=gen)}
        self.held = {k: torch.zeros_like(v) for k, v in self.new.items()}
        empty = lambda *s, t=kind: torch.empty(s, device="cuda", dtype=t)  # noqa: E731
        self.out = {"loss": empty(m, t=torch.float32), "lse": empty(m, t=torch.float32), "dX": empty(m, n), "dW": empty(p, n, t=torch.float32),
                    "one": empty(1, p), "few": empty(40, p), "many": empty(m, p), "back": empty(p, n)}
        self.room = torch.empty(max(lm.cross_entropy_workspace_bytes(m, n, p), lm.cross_entropy_workspace_bytes(m, n, p, True),
                                    lm.linear_workspace_bytes(m, n, p, "tile"), lm.linear_workspace_bytes(40, n, p, "shared")), dtype=torch.uint8, device="cuda")

    def run(self):
        lm, h, o = self.lm, self.held, self.out
        lm.cross_entropy(h["X"], h["W"], h["y"], loss=o["loss"], lse=o["lse"], workspace=self.room)
        lm.cross_entropy_backward(h["g"], h["X"], h["W"], h["y"], o["lse"], dX=o["dX"], dW=o["dW"], workspace=self.room)
        P = lm.quantize(h["W"], group=64, zeros=True)
        P = lm.pack(*lm.unpack(P), n=P.n, group=64)
        lm.linear(h["X"][:1], P, D=o["one"])
        lm.linear(h["X"][:40], P, D=o["few"], workspace=self.room, way="shared")
        lm.linear(h["X"], P, D=o["many"], workspace=self.room, way="tile")
        lm.dequantize(P, out=o["back"])

    def fill(self):
        for k, t in self.new.items():
            self.held[k].copy_(t)

    def clear(self):
        for t in self.out.values():
            t.fill_(float("nan"))
        self.room.fill_(255)
        for t in self.held.values():
            t.zero_()

    def results(self):
        return {k: t.clone() for k, t in self.out.items()}


SIZES = [(60, 256, 1000, torch.bfloat16), (300, 520, 1111, torch.float16)]


@pytest.mark.parametrize("m,n,p,kind", SIZES)
def test_another_stream_behind_long_work(lm, m, n, p, kind):
    step = Step(lm, m, n, p, kind, 1)
    step.fill()
    step.run()
    want = step.results()
    big = torch.randn((8192, 8192), device="cuda").bfloat16()
    stream = torch.cuda.Stream()
    for _ in range(3):
        step.clear()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for _ in range(8):
                big = torch.mm(big, big).mul_(2.0 ** -7)
            step.fill()
            step.run()
        torch.cuda.current_stream().wait_stream(stream)
        for k, t in step.out.items():
            assert torch.equal(t, want[k]) and torch.isfinite(t).all(), k
    torch.cuda.synchronize()


@pytest.mark.parametrize("m,n,p,kind", SIZES)
def test_graphs_that_share_a_workspace(lm, m, n, p, kind):
    steps = [Step(lm, m, n, p, kind, seed) for seed in (1, 2)]
    steps[1].room = steps[0].room
    want = []
    for s in steps:
        s.fill()
        s.run()
        want.append(s.results())
    torch.cuda.synchronize()
    graphs = []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    other = Step(lm, 50, 72, 130, kind, 3)
    other.fill()
    for i in range(4):
        for s in steps:
            s.clear()
        for s in steps:
            s.fill()
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        other.run()                                                  # (eager work of the program's own between replays)
        for s, w in zip(steps, want):
            for k, t in s.out.items():
                assert torch.equal(t, w[k]), (i, k)
        if i % 2:
            torch.cuda.synchronize()


def test_two_streams_at_once(lm):
    """With workspaces of their own."""
    steps = [Step(lm, 300, 264, 3000, torch.bfloat16, seed) for seed in (4, 5)]
    want = []
    for s in steps:
        s.fill()
        s.run()
        want.append(s.results())
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for st, s in zip(streams, steps):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                for _ in range(3):
                    s.run()
        for st in streams:
            torch.cuda.current_stream().wait_stream(st)
        for s, w in zip(steps, want):
            for k, t in s.out.items():
                assert torch.equal(t, w[k]), k
