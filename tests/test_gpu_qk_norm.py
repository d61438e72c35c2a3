"""Models with normed query and key heads through the engine, against the CPU oracle step by step."""
import numpy as np
import pytest
import torch

import paper_2504_00030_amd as pk
import synth
from paper_2504_00030_amd import binding
from parity_utils import TOL, run_lockstep, to_gpu

pytestmark = pytest.mark.gpu


def _with_norms(W, shape, seed):
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if shape.dtype == "fp32" else torch.bfloat16
    new = lambda: [(1.0 + 0.3 * torch.randn(shape.head_dim, generator=g)).to(dt) for _ in range(shape.n_layers)]
    return dict(W, q_norm=new(), k_norm=new())


def _models(cfg, which=("target", "draft")):
    Wt, Wd = synth.make_pair_weights(cfg, 3, norm_jitter=0.1)
    if "target" in which:
        Wt = _with_norms(Wt, cfg.target, 11)
    if "draft" in which:
        Wd = _with_norms(Wd, cfg.draft, 12)
    return Wt, Wd


def _engine(cfg, Wt, Wd, prompt_len, n_generate, batch, **kw):
    return pk.SpecEngine(cfg.target, to_gpu(Wt), cfg.draft, to_gpu(Wd), batch=batch,
                         max_seq=prompt_len + (n_generate + 2 * cfg.gamma_max + 4) * (4 if batch > 1 else 1),
                         gamma_max=cfg.gamma_max, **kw)


def _run(cfg, *, controller="gammatune", temperature=1.0, prompt_len=None, n_generate=24, batch=1, tau=0.0,
         which=("target", "draft"), **kw):
    prompt_len = prompt_len or cfg.prompt_len
    Wt, Wd = _models(cfg, which)
    eng = _engine(cfg, Wt, Wd, prompt_len, n_generate, batch, temperature=temperature, seed=5, **kw)
    if tau > 0:
        eng.set_early_stop(tau)
    prompts = synth.make_prompts(batch, prompt_len, cfg.target.vocab, 7)
    c = run_lockstep(eng, cfg, synth.to_numpy_weights(Wt), synth.to_numpy_weights(Wd), prompts, n_generate, controller=controller,
                     temperature=temperature, seed=5, tau=tau)
    eng.close()
    print(f"coverage {c.coverage:.3f} max logit err {c.max_logit_err:.3e}")
    assert not c.failures, "\n".join(c.failures[:10])
    assert c.max_logit_err <= TOL[cfg.target.dtype]
    assert c.coverage >= 0.8


@pytest.mark.parametrize("which", [("target", "draft"), ("target",), ("draft",)], ids=["both", "target", "draft"])
def test_tiny_fp32_pair(which):
    _run(synth.pair("tiny"), which=which)


@pytest.mark.parametrize("path", [0, 1, 2], ids=["auto", "wavedot", "mfma"])
def test_small_bf16_pair(path):
    _run(synth.pair("small-bf16"), gemv_path=path)


@pytest.mark.parametrize("pair", ["small-bf16-hd128", "small-q8", "small-q8-hd128"])
def test_other_small_pairs(pair):
    _run(synth.pair(pair), temperature=0.0, controller="fixed4")


@pytest.mark.parametrize("graphs", [True, False])
def test_batch_with_early_stopping(graphs):
    _run(synth.pair("small-bf16"), batch=3, tau=0.05, use_graphs=graphs, controller="spread", n_generate=16)


@pytest.mark.parametrize("page_tokens", [8, 16, 64])
def test_page_sizes(page_tokens):
    """Both arrangements inside a page (plain below 16 tokens, fragment order from there)."""
    _run(synth.pair("small-bf16"), page_tokens=page_tokens, temperature=0.0, n_generate=16)


def test_long_prompt_through_the_ingestion_kernels():
    _run(synth.pair("small-bf16"), prompt_len=1100, n_generate=8, temperature=0.0)


@pytest.mark.parametrize("pair_name,batch", [("1b", 1), ("8b", 3)])
def test_full_widths_at_reduced_depth(pair_name, batch):
    """The large pairs' widths, two target layers and one draft layer deep, drawn at a temperature in graphs."""
    from oracle import model as om
    cfg = synth.shrink(synth.pair(pair_name), 2, 1)
    Wt, Wd = synth.make_pair_weights(cfg, 0, device="cuda")
    cpu = lambda W: {k: W[k] for k in ("q_norm", "k_norm")}
    gpu = lambda W, extra: dict(W, **{k: [t.cuda() for t in v] for k, v in extra.items()})
    Wt, Wd = gpu(Wt, cpu(_with_norms({}, cfg.target, 1))), gpu(Wd, cpu(_with_norms({}, cfg.draft, 2)))
    torch.cuda.synchronize()
    widen = lambda W: {k: ([om.as_f64(a) for a in v] if isinstance(v, list) else om.as_f64(v))
                       for k, v in synth.to_numpy_weights(W).items()}
    eng = pk.SpecEngine(cfg.target, Wt, cfg.draft, Wd, batch=batch, max_seq=512, gamma_max=4, temperature=0.0, seed=0, use_graphs=True)
    prompts = synth.make_prompts(batch, 60, cfg.target.vocab, 7)
    c = run_lockstep(eng, cfg, widen(Wt), widen(Wd), prompts, 6, controller="fixed3", temperature=0.0, seed=0)
    eng.close()
    assert not c.failures, "\n".join(c.failures[:10])
    assert c.max_logit_err <= TOL["bf16"] and c.coverage >= 0.7


def test_switching_the_norms_on_and_off():
    """Without the norms again, the engine gives the bits it gave before; and a change asks for a new prompt."""
    cfg = synth.pair("small-bf16")
    Wt, Wd = synth.make_pair_weights(cfg, 3)
    eng = _engine(cfg, Wt, Wd, 40, 24, 1, temperature=0.0, seed=5, use_graphs=True)
    prompts = synth.make_prompts(1, 40, cfg.target.vocab, 7)

    def steps():
        eng.prefill(prompts)
        out = []
        for _ in range(3):
            eng.draft(3)
            eng.verify(3)
            q = eng.debug_logits(0)
            out.append((q, eng.accept(), eng.debug_logits(1)))
        return out

    def same(a, b):
        return all(np.array_equal(x[0], y[0]) and np.array_equal(x[2], y[2]) for x, y in zip(a, b))

    before = steps()
    Wn = to_gpu(_with_norms(Wt, cfg.target, 11))
    for _ in range(2):
        eng.set_qk_norm(1, Wn["q_norm"], Wn["k_norm"])
        with pytest.raises(pk.SpecError) as e:
            eng.draft(3)
        assert e.value.code == binding.SPEC_ESTATE
        normed = steps()
        assert not same(before, normed)
        held = eng.device_bytes()
        eng.set_qk_norm(1, None, None)
        with pytest.raises(pk.SpecError):
            eng.draft(3)
        assert same(before, steps())
    eng.set_qk_norm(1, Wn["q_norm"], Wn["k_norm"])
    assert same(normed, steps()) and eng.device_bytes() == held
    eng.close()


def test_refusals():
    cfg = synth.pair("small-bf16")
    Wt, Wd = synth.make_pair_weights(cfg, 3)
    eng = _engine(cfg, Wt, Wd, 40, 8, 1, temperature=0.0)
    good = [torch.ones(cfg.target.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(cfg.target.n_layers)]
    for q, k in ((good, good[:-1]), (good, [t.float() for t in good]), ([t[:8] for t in good], good), ([t.cpu() for t in good], good)):
        with pytest.raises(ValueError):
            eng.set_qk_norm(1, q, k)
    for q, k in ((good, None), (None, good)):
        with pytest.raises(pk.SpecError) as e:
            eng.set_qk_norm(1, q, k)
        assert e.value.code == binding.SPEC_EINVAL
    assert eng._lib.spec_set_qk_norm(eng._ctx, 2, None, None) == binding.SPEC_EINVAL
    assert eng._lib.spec_set_qk_norm(None, 1, None, None) == binding.SPEC_EINVAL
    eng.close()


@pytest.mark.parametrize("model", [-1, 2])
def test_norms_of_no_model_are_refused(model):
    cfg = synth.pair("tiny")
    Wt, Wd = synth.make_pair_weights(cfg, 3)
    eng = _engine(cfg, Wt, Wd, 16, 8, 1)
    g = [torch.ones(cfg.target.head_dim, device="cuda") for _ in range(cfg.target.n_layers)]
    with pytest.raises(ValueError, match="model"):
        eng.set_qk_norm(model, g, g)
    with pytest.raises(pk.SpecError):
        eng.set_qk_norm(model, None, None)
    eng.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd_target,hd_draft", [(256, 24), (512, 8), (136, 48)])
def test_other_head_sizes(dtype, hd_target, hd_draft):
    """Heads of 8 to 512 elements, whole lanes' worth and not, through the plain and the re-tiled projections."""
    from synth.configs import ModelShape, PairConfig
    target = ModelShape(2, 64, 2, 1, hd_target, 128, 512, 10000.0, 1e-5, dtype)
    draft = ModelShape(2, 64, 4, 2, hd_draft, 128, 512, 10000.0, 1e-5, dtype)
    _run(PairConfig("heads", target, draft, "independent", 40, 16, 8), n_generate=12, temperature=0.0, controller="fixed4")


@pytest.mark.parametrize("pair", ["tiny", "small-bf16"])
def test_the_norm_kernel_is_timed(pair):
    """Class 8 of the kernel timing: one launch a layer and pass in models with normed heads, none in the others."""
    cfg = synth.pair(pair)
    Wt, Wd = _models(cfg, which=("target",))
    eng = _engine(cfg, Wt, Wd, 17, 8, 1, temperature=0.0)
    eng.prefill(synth.make_prompts(1, 17, cfg.target.vocab, 7))
    for kind in (0, 8):
        eng.profile_kernel(1, kind)
        eng.draft(3)
        eng.verify(3)
        eng.accept()
        launches, ms = eng.profile_read_class(1, 8)
        assert launches == cfg.target.n_layers and ms > 0
        assert eng.profile_read_class(0, 8)[0] == 0
        if kind == 0:
            assert eng.profile_read_class(1, 1)[0] == cfg.target.n_layers * (3 if pair == "tiny" else 1)
            assert eng.profile_read_class(0, 1)[0] == 3 * cfg.draft.n_layers
        total, ms_total = eng.profile_read()
        assert total >= launches and ms_total >= ms
    with pytest.raises(pk.SpecError):
        eng.profile_kernel(1, 9)
    eng.close()
