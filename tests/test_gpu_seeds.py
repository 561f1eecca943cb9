"""The sampler, AdamW's rounding and dropout draw from one generator: what keeps their bits apart."""
import pytest
import torch

from oracle import train_oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import Context
    c = Context(0)
    yield c
    c.close()


def test_by_default_dropout_does_not_drop_by_the_bits_that_round(ctx):
    n, t, tensor = 1 << 14, 3, 0
    w = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    step = ctx.make_adamw_step([w], [w.clone()], **ctx.adamw_state([w], 8))
    kept = ctx.gg_dropout(torch.ones(1, n, device="cuda"), 0.5, t, tensor_id=tensor)["y"][0].cpu() != 0
    rounds_up = torch.from_numpy(train_oracle.rounding_noise(n, t, tensor, step.args.seed).reshape(-1)[:n] >= 32768)
    # independent bits agree in half of the places, 5 standard deviations around it; the same bits in all
    assert abs((kept == rounds_up).double().mean().item() - 0.5) <= 5 * 0.5 / n ** 0.5


def test_a_training_run_gives_each_draw_a_seed_of_its_own(ctx, monkeypatch):
    from paper_2506_00486_b200 import Context
    from paper_2506_00486_b200.train_example import train_tokens
    seen = {"dropout": set(), "rounding": set(), "weights": set()}
    sample, dropout, adamw = Context.gg_sample, Context.make_dropout, Context.make_adamw_step

    def note_sample(self, out, beta, alpha, seed, *a, **kw):
        seen["weights"].add(seed)
        return sample(self, out, beta, alpha, seed, *a, **kw)

    def note(kind, make):
        def wrapped(*a, **kw):
            made = make(*a, **kw)
            seen[kind].add(made.args.seed)
            return made
        return wrapped

    monkeypatch.setattr(Context, "gg_sample", note_sample)
    monkeypatch.setattr(Context, "make_dropout", note("dropout", dropout))
    monkeypatch.setattr(Context, "make_adamw_step", note("rounding", adamw))
    losses, _, _ = train_tokens(ctx, steps=2)
    assert torch.isfinite(losses).all()
    assert all(len(s) == 1 for s in seen.values()) and len(set.union(*seen.values())) == 3
