"""Tokens drawn from a step's mixture (dbt_sample_last) against the 64-bit forms of the mixture and of the sampler, on the
logits and alpha that the same step hands out."""
import numpy as np
import pytest
import torch

import ref_drafts as ref
from gpu_util import library
from paper_2608_12385_b200 import binding
from paper_2608_12385_b200.inputs import ModelConfig, make_tokens, make_weights

pytestmark = pytest.mark.gpu

DENSE = ModelConfig(d_model=256, n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, d_ff=704, vocab=5000, weight_dtype="bf16")
CONFIGS = {
    "bf16": DENSE,
    "bf16-4-paths": DENSE.replace(n_paths=4),
    "fp32": DENSE.replace(weight_dtype="fp32", vocab=900),
    "moe": DENSE.replace(n_experts=8, d_expert=128, n_shared_experts=1, k_primary=2, k_branch=2, d_ff=0),
}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    library()


def model(cfg, B):
    return binding.Model(cfg, binding.weights_to_device(make_weights(cfg, seed=0, matrix_std=0.08), "cuda:0"), B, 64)


def mixture_scores(out):
    z1, z2, alpha = (out[k].double().cpu() for k in ("z1", "z2", "alpha"))
    q = torch.softmax(z2, dim=-1)
    return torch.log(alpha[:, None] * torch.softmax(z1, dim=-1) + (1 - alpha[:, None]) * (q.mean(0) if q.dim() == 3 else q)).numpy()


def check(scores, drawn, u, kw, B):
    """Scores are fp32 logarithms of sums of exponentials and quotients of fp32: off by at most 2^-18 where they are above -80 (an
    exponential's argument of at most 80 in fp32 is off by 2^-18, the rest is below that).  A running sum moves by no more, relative; a
    token has to be the 64-bit form's unless a decision is closer than that."""
    tok, lp = drawn[0].cpu().tolist(), drawn[1].cpu().tolist()
    sure = 0
    for b in range(B):
        at = lambda k, d: d if k not in kw else float(kw[k][b])  # noqa: E731
        want, logp, near = ref.sample_row(scores[b], float(np.float32(u[b])), at("temperature", 1.0), int(at("top_k", 0)), at("top_p", 1.0), at("min_p", 0.0))
        t = at("temperature", 1.0)
        if near < 2.0 ** -16 / max(min(t, 1.0), 0.1):
            continue
        if at("top_k", 0) > 0:  # the border of top-k: two scores closer than their error may change places
            z = np.sort(scores[b])[::-1]
            if z[int(at("top_k", 0)) - 1] - z[int(at("top_k", 0))] < 2.0 ** -16:
                continue
        sure += 1
        assert tok[b] == want, (b, tok[b], want, near)
        assert abs(lp[b] - logp) <= 2.0 ** -14 / max(min(t, 1.0), 0.1)
    return sure


@pytest.mark.parametrize("name", sorted(CONFIGS))
def test_sampling_from_the_mixture(name):
    cfg, B = CONFIGS[name], 4
    m = model(cfg, B)
    tok = make_tokens(cfg, B, 12, seed=1).cuda()
    m.prefill(tok[:, :8].contiguous())
    g = torch.Generator().manual_seed(5)
    sure = 0
    for t in range(8, 12):
        out = m.decode_full(tok[:, t].contiguous())
        scores = mixture_scores(out)
        for kw in ({}, dict(temperature=[0.7] * B), dict(top_k=[5, 40, 0, 300], top_p=[0.9] * B), dict(min_p=[0.05] * B, temperature=[1.3] * B)):
            u = torch.rand(B, generator=g)
            dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32).cuda() for k, v in kw.items()}
            sure += check(scores, m.sample_last(u.cuda(), **dev), u.tolist(), kw, B)
        greedy = m.sample_last(torch.zeros(B, device="cuda"), temperature=torch.zeros(B, device="cuda"))[0]
        gap = np.sort(scores, axis=1)[:, ::-1]
        for b in range(B):
            if gap[b, 0] - gap[b, 1] > 2.0 ** -16:
                assert int(greedy[b]) == int(out["next"][b])
    assert sure >= 40  # most draws are decided
    assert m.sync_status() == (0, 0)


@pytest.mark.parametrize("name", ["bf16", "bf16-4-paths", "fp32"])
@pytest.mark.parametrize("temperature", [1.0, 20.0, 80.0])
def test_temperature_reaches_tokens_whose_probability_fp32_does_not_hold(name, temperature):
    """Logits spread over some hundred, so that most probabilities are below the smallest number of fp32, while the temperature gives their
    tokens most of the mass.

    Every logit stands twice, so alpha is 0.5.  A score is a sum of a difference of logits (below 2^10 here), logarithms of sums and of alpha, and
    one more logarithm: four roundings of at most 2^-15 each, and the sums' own 2^-19: below 2^-12.  The mass of a set moves by 2^-12 / T
    relative, in numerator and denominator."""
    cfg, B = CONFIGS[name], 4
    weights = make_weights(cfg, seed=0, matrix_std=0.08)
    head = weights["lm_head"]
    half = cfg.vocab // 2
    head[half:2 * half] = head[:half]
    m = binding.Model(cfg, binding.weights_to_device(weights), B, 64)
    tok = make_tokens(cfg, B, 12, seed=1).cuda()
    spread = float(m.decode_full(tok[:, 0].contiguous())["z1"].std())
    weights["lm_head"] = (head.float() * (60.0 / spread)).to(head.dtype)
    m = binding.Model(cfg, binding.weights_to_device(weights), B, 64)
    g, sure, far = torch.Generator().manual_seed(8), 0, 0
    bound = 2 * 2.0 ** -12 / temperature
    for t in range(12):
        out = m.decode_full(tok[:, t].contiguous())
        assert (out["alpha"] - 0.5).abs().max() <= 2.0 ** -20
        scores = mixture_scores(out)
        assert 150 < -scores.min() < 2 ** 10
        u = torch.rand(B, generator=g)
        drawn, logp = (x.tolist() for x in m.sample_last(u.cuda(), temperature=torch.full((B,), temperature, device="cuda")))
        for b in range(B):
            want, lp, near = ref.sample_row(scores[b], float(u[b]), temperature)
            if near > bound:
                sure += 1
                far += scores[b][want] < -110
                assert drawn[b] == want, (drawn[b], want, near)
                assert abs(logp[b] - lp) <= bound + 2.0 ** -20
    assert sure >= 24
    assert temperature < 80 or far >= 12


def test_sampling_after_primary_only_and_boundary_steps():
    cfg, B = CONFIGS["bf16"], 3
    m = model(cfg, B)
    tok = make_tokens(cfg, B, 10, seed=2).cuda()
    u = torch.rand(B, generator=torch.Generator().manual_seed(6))
    out = m.prefill_boundary(tok[:, :9].contiguous())
    assert check(mixture_scores(out), m.sample_last(u.cuda()), u.tolist(), {}, B) >= 1
    out = m.decode_full(tok[:, 9].contiguous(), grouped=False)
    drawn = m.sample_last(u.cuda(), top_k=torch.full((B,), 20, dtype=torch.int32, device="cuda"))
    want = [ref.sample_row(out["z1"][b].cpu().numpy(), float(u[b]), top_k=20) for b in range(B)]
    assert drawn[0].tolist() == [w[0] for w in want]  # the logits themselves: exact


def test_sampled_decoding_feeds_itself_and_leaves_the_cache_as_greedy_steps_do():
    """The drawn token written straight into the next step's input; the cache holds what teacher-forced steps write."""
    cfg, B = CONFIGS["bf16"], 2
    m, n = model(cfg, B), model(cfg, B)
    tok = make_tokens(cfg, B, 5, seed=3).cuda()
    for x in (m, n):
        x.prefill(tok[:, :4].contiguous())
    cur, g, fed = tok[:, 4].contiguous(), torch.Generator().manual_seed(7), []
    for _ in range(10):
        fed.append(cur.clone())
        m.decode_step(cur)
        m.sample_last(torch.rand(B, generator=g).cuda(), top_p=torch.full((B,), 0.9, device="cuda"), next_dev=cur)
    for t in fed:
        n.decode_step(t.clone())
    for a, b in zip(m.export_kv(B, 14), n.export_kv(B, 14)):
        assert torch.equal(a, b)
    assert len({int(t[0]) for t in fed}) > 3


@pytest.mark.parametrize("own", [True, False])
def test_a_model_on_another_stream_than_the_callers(own):
    """The model on a stream of its own and the caller on the default one, or the other way round.  While the model's stream is still
    busy, memory of a dropped result or input goes to nobody who works on the caller's stream, and all results are those of one stream."""
    cfg, B = CONFIGS["bf16"], 4
    side = torch.cuda.Stream()
    weights = binding.weights_to_device(make_weights(cfg, seed=0, matrix_std=0.08), "cuda:0")
    tok = make_tokens(cfg, B, 9, seed=9).cuda()
    u, p = torch.rand(B, generator=torch.Generator().manual_seed(10)), torch.full((B,), 0.9)
    plain = binding.Model(cfg, weights, B, 64)
    logits, first = plain.prefill(tok[:, :4].contiguous(), want_logits=True), plain.prefill_boundary(tok[:, 4:].contiguous())
    want = plain.sample_last(u.cuda(), top_p=p.cuda())
    m = binding.Model(cfg, weights, B, 64, stream=side if own else None)
    models, callers = (side, torch.cuda.default_stream()) if own else (torch.cuda.default_stream(), side)
    with torch.cuda.stream(callers):
        a, b = tok[:, :4].contiguous(), tok[:, 4:].contiguous()
        torch.cuda.synchronize()
        got_logits, got = m.prefill(a, want_logits=True), m.prefill_boundary(b)
        du, dp, _ = u.cuda(), p.cuda(), torch.full((B,), 7.0, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(models):
            torch.cuda._sleep(600_000_000)  # a third of a second
        busy = torch.cuda.Event()
        tokens, logp = m.sample_last(du, top_p=dp)
        busy.record(models)
        gone = {x.data_ptr() for x in (logp, du, dp)}
        del logp, du, dp
        others = [torch.full((B,), 7.0, device="cuda") for _ in range(600)]
        assert not busy.query()  # the sampler has yet to run
        assert not gone & {x.data_ptr() for x in others}
        kept, logp = m.sample_last(u.cuda(non_blocking=False), top_p=p.cuda())
        torch.cuda.synchronize()
        assert all((x == 7.0).all() for x in others)
        for x, y in ((tokens, want[0]), (kept, want[0]), (logp, want[1]), (got_logits, logits), *((got[k], first[k]) for k in first)):
            assert torch.equal(x, y)


def test_refusals():
    cfg, B = CONFIGS["fp32"], 2
    m = model(cfg, B)
    tok, u = make_tokens(cfg, B, 4, seed=4).cuda(), torch.zeros(B, device="cuda")
    for prepare, status in ((lambda: None, 4), (lambda: m.prefill(tok[:, :3].contiguous()), 4)):
        prepare()
        with pytest.raises(binding.DbtError) as e:
            m.sample_last(u)
        assert e.value.status == status
    m.decode_full(tok[:, 3].contiguous())
    m.sample_last(u)
    for bad in (lambda: m.sample_last(torch.zeros(1, device="cuda")), lambda: m.sample_last(u, top_k=u), lambda: m.sample_last(u.cpu())):
        with pytest.raises(binding.DbtError) as e:
            bad()
        assert e.value.status == 1
    m.reset()
    with pytest.raises(binding.DbtError) as e:
        m.sample_last(u)
    assert e.value.status == 4
