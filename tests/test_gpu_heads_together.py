"""The operators as they are used together: a student's head and its features' norm
learn from a teacher's best classes; a policy's step; and where two operators say the
same thing, that they agree.

Tolerances. Each operator's output is within 2^-18 of the size of its terms (FP32; the
operators' own tests), and each hands on what the one before left: five in a row, whose
sums over features and classes of either sign let errors stand at most 2^4 out of the
sums' size here, are within 5 2^-18 2^4 < 2^-11 of the result's norm.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NEAR = 2.0 ** -11


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    return torch.device("cuda", 0)


@pytest.fixture(scope="module")
def heads(dev):
    from paper_2608_13144_gb300 import heads
    yield heads
    assert heads.operator_errors(dev) == 0


def near(got, want, what):
    got, want = got.detach().cpu().double(), want.detach().cpu().double()
    assert got.shape == want.shape
    assert float((got - want).norm()) <= NEAR * float(want.norm()), what


def setting(dev, n=300, d=96, c=130, g=4, r=6, k=12):
    gen = torch.Generator().manual_seed(7)
    def rnd(*s):
        return torch.randn(*s, generator=gen)
    t = dict(x=rnd(n, d) * 2 + 1, weight=1 + 0.2 * rnd(d), bias=0.1 * rnd(d), W=rnd(c, d) / d ** 0.5,
             A=rnd(g, r, d) / d ** 0.5, B=rnd(g, c, r) / r ** 0.5, head_bias=0.1 * rnd(c), teacher=2 * rnd(n, c),
             row=torch.rand(n, generator=gen) / n)
    ids = torch.randint(-1, g, (n,), generator=gen).int()
    return {name: v.to(dev) for name, v in t.items()}, ids.to(dev), k


def student_step(heads, t, ids, k, T=2.0):
    """(loss, dx, dweight, dbias, dA, dB) of one distillation step."""
    best = heads.log_probs(t["teacher"], top=k)
    y, stats = heads.layer_norm(t["x"], t["weight"], t["bias"])
    z = heads.adapted_logits(y, t["W"], t["A"], t["B"], ids, t["head_bias"])
    loss, dz = heads.distill(z, best.top, best.index, t["row"], temperature=T, in_place=True)
    dy, dA, dB = heads.adapted_logits_backward(dz, y, t["W"], t["A"], t["B"], ids)
    return (loss, *heads.layer_norm_backward(dy, t["x"], stats, t["weight"]), dA, dB)


def student_logits(v, ids):
    """The student's logits in 64 bits, for autograd."""
    y = torch.nn.functional.layer_norm(v["x"], v["x"].shape[1:], v["weight"], v["bias"], 1e-5)
    z = y @ v["W"].t() + v["head_bias"]
    low = torch.einsum("grd,nd->ngr", v["A"], y)
    all_ = torch.einsum("gcr,ngr->ngc", v["B"], low)
    pick = torch.nn.functional.one_hot(ids.clamp(min=0), len(v["A"])).double() * (ids >= 0)[:, None]
    return z + (all_ * pick[:, :, None]).sum(1)


def leaves(t):
    v = {name: x.cpu().double() for name, x in t.items()}
    for name in ("x", "weight", "bias", "A", "B"):
        v[name].requires_grad_()
    return v


def test_a_student_learns_from_a_teacher(dev, heads):
    t, ids, k = setting(dev)
    T = 2.0
    got = student_step(heads, t, ids, k, T)
    v, rows = leaves(t), ids.cpu().long()
    best = torch.sort(v["teacher"], dim=1, descending=True, stable=True)
    q = torch.softmax(best.values[:, :k] / T, 1)
    lp = torch.log_softmax(student_logits(v, rows) / T, 1).gather(1, best.indices[:, :k])
    loss = v["row"] * T * T * (q * (torch.log(q) - lp)).sum(1)
    loss.sum().backward()
    want = (loss, v["x"].grad, v["weight"].grad, v["bias"].grad, v["A"].grad, v["B"].grad)
    for name, a, b in zip(("loss", "dx", "dweight", "dbias", "dA", "dB"), got, want):
        near(a, b, name)


def test_a_policy_step(dev, heads):
    t, ids, _ = setting(dev)
    n, c = t["teacher"].shape
    gen = torch.Generator().manual_seed(3)
    target = torch.randint(0, c, (n,), generator=gen)
    gain = torch.randn(n, generator=gen).double()
    y, stats = heads.layer_norm(t["x"], t["weight"], t["bias"])
    z = heads.adapted_logits(y, t["W"], t["A"], t["B"], ids, t["head_bias"])
    to = target.int().to(dev)
    r = heads.log_probs(z, to, temperature=0.7)
    dz = heads.log_probs_backward(z, r.norm, to, gain.float().to(dev), torch.full((n,), 0.01, device=dev), temperature=0.7,
                                  in_place=True)
    dy, dA, dB = heads.adapted_logits_backward(dz, y, t["W"], t["A"], t["B"], ids)
    got = (r.logprob, r.entropy, *heads.layer_norm_backward(dy, t["x"], stats, t["weight"]), dA, dB)
    v = leaves(t)
    lp = torch.log_softmax(student_logits(v, ids.cpu().long()) / 0.7, 1)
    given, entropy = lp.gather(1, target[:, None])[:, 0], -(lp.exp() * lp).sum(1)
    (gain * given + 0.01 * entropy).sum().backward()
    want = (given, entropy, v["x"].grad, v["weight"].grad, v["bias"].grad, v["A"].grad, v["B"].grad)
    for name, a, b in zip(("logprob", "entropy", "dx", "dweight", "dbias", "dA", "dB"), got, want):
        near(a, b, name)


def test_a_step_in_a_graph(dev, heads):
    """Captured and replayed on other features, while an eager step runs on another stream."""
    t, ids, k = setting(dev)
    want = student_step(heads, t, ids, k)
    held = {name: torch.ones_like(v) for name, v in t.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = student_step(heads, held, ids, k)
    for name, v in t.items():
        held[name].copy_(v)
    torch.cuda.synchronize()
    side = torch.cuda.Stream(dev)
    with torch.cuda.stream(side):
        beside = student_step(heads, t, ids, k)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, e in zip(want, got, beside):
        assert torch.equal(a, b) and torch.equal(a, e)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c", [50, 700, 12_000])
def test_where_operators_say_the_same(dev, heads, dtype, c):
    """Cross entropy is minus the log-probability, and what distillation from one class or from a certain teacher says."""
    gen = torch.Generator().manual_seed(c)
    z = (3 * torch.randn(40, c, generator=gen)).to(dtype).to(dev)
    y = torch.randint(0, c, (40,), generator=gen).int().to(dev)
    w = torch.rand(40, generator=gen).to(dev)
    loss, dz = heads.cross_entropy(z, y, w)
    r = heads.log_probs(z, y, top=2)
    scored = heads.log_probs_backward(z, r.norm, y, -w)
    one, from_one = heads.distill(z, torch.zeros(40, 1, device=dev), y[:, None].contiguous(), w)
    other = ((y + 1) % c).int()
    two, from_two = heads.distill(z, torch.tensor([[0.0, -200.0]], device=dev).expand(40, 2), torch.stack([y, other], 1), w)
    near(-w * r.logprob, loss, "logprob")
    for a, b in ((one, loss), (two, loss), (scored, dz), (from_one, dz), (from_two, dz)):
        if a.dtype == torch.bfloat16:  # two roundings of values that differ in their last bits: a step of BF16
            assert ((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 1e-12).all()
        else:
            near(a, b, "same")
    # the best class's log-probability is that of the largest logit's cross entropy
    top = heads.cross_entropy(z, r.index[:, 0].contiguous(), need_grad=False)[0]
    near(-r.top[:, 0], top, "top")
