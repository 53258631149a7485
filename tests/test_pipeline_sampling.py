"""Sampled generation through the shard pipeline: the drawn tokens are those the definition gives for every pass's own
logits, under every schedule, and they are what the next iteration consumes."""
from types import SimpleNamespace

import pytest
import torch

from tests import kv8_reference as R


def _fake_shards(head=True):
    stream = SimpleNamespace(cuda_stream=1, device=torch.device("cpu"))
    return [SimpleNamespace(stream=stream, layer_end=2 if head else 1, desc=SimpleNamespace(n_layers_total=2))]


def test_sampling_arguments_are_checked_at_construction():
    from paper_2405_14371_b200.pipeline import ShardPipeline

    u, t = torch.rand(3, 2, 4), torch.ones(2, 4)
    ok = ShardPipeline(_fake_shards(), [[0] * 4, [1] * 4], 4, "sequential", sampling={"u": u, "temperature": t})
    assert tuple(ok.logprobs.shape) == (2, 4)
    for bad in ({"temperature": t}, {"u": u, "topk": t}, {"u": u[0]}, {"u": u, "top_p": t[:1]}, {"u": u[:, :, :3]}):
        with pytest.raises(ValueError):
            ShardPipeline(_fake_shards(), [[0] * 4, [1] * 4], 4, "sequential", sampling=bad)
    with pytest.raises(ValueError):
        ShardPipeline(_fake_shards(head=False), [[0] * 4, [1] * 4], 4, "sequential", sampling={"u": u})
    ok.iteration = 1
    with pytest.raises(RuntimeError):
        ok.decode(3)


@pytest.mark.gpu
def test_sampled_generation_matches_the_definition_under_every_schedule():
    from paper_2405_14371_b200 import binding as B
    from paper_2405_14371_b200.pipeline import ShardPipeline
    from tests.helpers import device_weights, slice_weights
    from workload import TINY, prompt_ids

    MB, T, S, batch = 3, 9, 5, 2
    wd, _ = device_weights(0, TINY, 0, TINY.n_layers)
    ids = prompt_ids(0, MB * batch, T, TINY.vocab, seed=5).cuda().reshape(MB, batch, T)
    g = torch.Generator().manual_seed(4)
    u = torch.rand(S + 1, MB, batch, generator=g).cuda()
    temperature = torch.tensor([[0.7, 1.3], [0.0, 1.0], [2.0, 0.5]]).cuda()
    top_k = torch.tensor([[0, 20], [5, 0], [100, 3]], dtype=torch.int32).cuda()
    top_p = torch.tensor([[0.9, 1.0], [1.0, 0.5], [0.95, 1.0]]).cuda()
    min_p = torch.full((MB, batch), 0.01).cuda()

    def run(schedule, sampling):
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        if schedule == "sequential":
            streams[1] = streams[0]
        kw = dict(max_slots=MB * batch, max_seq=T + S + 1, max_tokens=batch * T, max_batch=batch, kv_page_tokens=16)
        shards = [B.Shard(TINY, a, a + 1, slice_weights(wd, TINY, a, a + 1), stream=st, **kw) for a, st in zip((0, 1), streams)]
        pipe = ShardPipeline(shards, [[batch * m + i for i in range(batch)] for m in range(MB)], batch, schedule, sampling=sampling)
        got = {}

        def keep(p, out):
            got[p] = (out[1].clone(), out[2].clone(), pipe.tokens[p.micro_batch].clone(), pipe.logprobs[p.micro_batch].clone())

        pipe.prefill(ids, T, on_output=keep)
        pipe.decode(S, on_output=keep)
        pipe.join(torch.cuda.current_stream())
        torch.cuda.synchronize()
        for sh in shards:
            sh.es_shard_device_status()
            sh.close()
        return got

    settings = {"u": u, "temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p}
    ref = run("sequential", settings)
    assert len(ref) == MB * (S + 1)
    for p, (logits, greedy, tokens, logprobs) in ref.items():
        for i in range(batch):
            at = lambda t: float(t[p.micro_batch, i])  # noqa: E731
            want, logp = R.sample(logits[i].cpu(), float(u[p.iteration, p.micro_batch, i]), at(temperature), int(at(top_k)), at(top_p), at(min_p))
            assert int(tokens[i]) == want
            assert abs(float(logprobs[i]) - logp) <= 2.0 ** -24 * abs(logp) + 2.0 ** -26
        if p.micro_batch == 1:
            assert int(tokens[0]) == int(greedy[0])               # temperature 0
    assert any(int(t[0]) != int(g[0]) for _, g, t, _ in ref.values())
    for schedule in ("bubbles", "no_bubbles"):
        got = run(schedule, settings)
        assert got.keys() == ref.keys()
        for p in ref:
            for a, b in zip(ref[p], got[p]):
                assert torch.equal(a, b), (schedule, p)
    # with the settings that leave only the first token, sampling is greedy feedback
    greedy = run("sequential", None)
    one = run("sequential", {"u": u, "top_k": torch.ones(MB, batch, dtype=torch.int32).cuda()})
    for p in greedy:
        assert torch.equal(one[p][2], greedy[p][1]) and torch.equal(one[p][0], greedy[p][0])
