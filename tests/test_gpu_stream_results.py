"""Results that a call allocates itself, on a stream that is not the current one: they are not memory that the current stream
still writes to."""
import pytest

from paper_2006_11751_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["step", "step_indexed", "unroll", "loss"])
def test_results_are_not_what_the_current_stream_still_writes_to(torch_cuda, name):
    torch = torch_cuda
    from paper_2006_11751_amd import binding
    net = wl.network(0)
    pol = binding.Policy(net, wl.weights(net), max_batch=2 * net["B"])
    d, B = pol.device, net["B"]
    obs, done = (torch.from_numpy(f(net, 0)).to(d) for f in (wl.observations, wl.done_mask))
    h = torch.from_numpy(wl.initial_state(net)).to(d)
    tables, ids = [h.repeat(2, 1) for _ in range(2)], torch.arange(B, dtype=torch.int32, device=d)
    steps = [torch.stack([a, a]) for a in (obs, done)]
    hp = wl.loss_config((5, 4), 32, 64)
    tr = {k: torch.from_numpy(v).to(d) for k, v in wl.trajectories(hp, 6031).items()}
    call = {"step": lambda s: pol.step(obs, h, done, 7, 1, stream=s), "loss": lambda s: binding.appo_loss(hp, tr, stream=s),
            "step_indexed": lambda s: pol.step_indexed(obs, tables.pop(), ids, done, 7, 1, stream=s),
            "unroll": lambda s: pol.unroll(steps[0], h, steps[1], stream=s)}[name]
    want = call(None)
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device=d)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for _ in range(10):  # the current stream is behind with its work, and lets go of what it will write to
        busy @ busy
    for t in want.values():
        if t is not None:
            torch.full((2 * t.numel() * t.element_size(),), 255, dtype=torch.uint8, device=d)
            torch.full_like(t, 1)
    got = call(side)
    torch.cuda.synchronize()
    for n, t in want.items():
        assert n == "workspace" or torch.equal(got[n], t), n
    pol.close()
