"""The serving loop over the paged cache: pruned prompt, next turn and replayed decode steps."""
import numpy as np
import pytest
import torch

from oracle import pace_oracle as O

pytestmark = pytest.mark.gpu

NEW = [37, 5, 0, 130]        # kept tokens of the first call
TURN = [1, 40, 3, 0]         # of the second
STEPS = 20                   # crosses blocks of 16 slots and pages of 32
HQ, HKV, D = 14, 2, 64


@pytest.fixture(scope="module")
def serve():
    from paper_2608_27206_gb300 import build
    build.build()
    from paper_2608_27206_gb300 import pace as P
    from paper_2608_27206_gb300 import serve as S
    P.pace_init(0)
    P.pace_device_status(clear=True)
    yield S
    assert P.pace_device_status(clear=True)[0] == 0


def _tokens(seed, n, heads):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n, heads, D, generator=g).to(torch.bfloat16).cuda()


def _cu(n):
    return [int(x) for x in np.concatenate([[0], np.cumsum(n)])]


def run(S, window, sinks, graph):
    """The layer, the outputs of its calls and the last step's queries."""
    layer = S.ServeLayer(len(NEW), 200, page_size=32, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, max_positions=400, window=window,
                         sinks=sinks)
    n = 2 * sum(NEW)
    rows = torch.from_numpy(np.sort(np.random.default_rng(1).permutation(n)[:sum(NEW)]).astype(np.int32)).cuda()
    ids = torch.randint(0, 400, (3, n), generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    outs = [layer.prompt(_tokens(3, n, HKV), _tokens(4, n, HKV), _tokens(5, n, HQ), _cu(NEW), ids, rows=rows)]
    m = sum(TURN)
    outs.append(layer.prompt(_tokens(6, m, HKV), _tokens(7, m, HKV), _tokens(8, m, HQ), _cu(TURN), ids[:, :m].contiguous()))
    k, v, q = _tokens(9, 4, HKV), _tokens(10, 4, HKV), _tokens(11, 4, HQ)
    pos = ids[:, m:m + 4].contiguous()
    g = layer.capture_step(k, v, q, pos) if graph else None
    for i in range(STEPS):
        k.copy_(_tokens(20 + i, 4, HKV)), v.copy_(_tokens(50 + i, 4, HKV)), q.copy_(_tokens(80 + i, 4, HQ))
        pos.copy_((pos + 1) % 400)
        if graph:
            g.replay()
        else:
            layer.step(k, v, q, pos)
        outs.append(layer.out.clone())
    return layer, outs


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_loop(serve, window, sinks):
    layer, outs = run(serve, window, sinks, graph=False)
    lens = [a + b + STEPS for a, b in zip(NEW, TURN)]
    assert layer.lens.tolist() == lens
    # replays give what the calls give, bit for bit, results and cache
    other, again = run(serve, window, sinks, graph=True)
    assert other.lens.tolist() == lens
    for a, b in zip(outs, again):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    codes = {}
    for name in ("k", "v"):
        x, y = getattr(layer.cache, name).view(torch.uint8).cpu(), getattr(other.cache, name).view(torch.uint8).cpu()
        s, r = getattr(layer.cache, name + "_scale").cpu(), getattr(other.cache, name + "_scale").cpu()
        for b, n in enumerate(lens):
            for p in range(-(-n // 32)):
                page, used = int(layer.table[b, p]), min(32, n - 32 * p)
                assert torch.equal(x[page, :, :used], y[page, :, :used])
                assert torch.equal(s[page, :, :-(-used // 16)], r[page, :, :-(-used // 16)])
        codes[name] = (O.e4m3_values()[x.numpy()], s.numpy().astype(np.float64))
    # the last step against the oracle, from what the cache holds
    q = layer.q.float().cpu().numpy().astype(np.float64)
    got = outs[-1].float().cpu().numpy().astype(np.float64)
    for b, n in enumerate(lens):
        pages = layer.table[b].cpu().numpy()
        k, v = (O.kv_read(*codes[name], pages, n) for name in ("k", "v"))
        r = O.kv_attention(q[b:b + 1], k, v, O.kv_visible(n, 1, window, sinks), D ** -0.5)
        # bf16 rounding and weights of 8 bits, twice over; a score's sum of D products in fp32
        score = 2.0 ** -23 * (D + 8) * r["abs_score"] + 2.0 ** -20
        tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -8 + 2 * score[..., None]) * r["abs_out"] + 2.0 ** -17 * r["peak"][..., None]
        assert np.all(np.abs(got[b:b + 1] - r["out"]) <= tol)


def test_example(serve, capsys):
    serve.main(["--visual", "400", "--steps", "40"])
    said = capsys.readouterr().out
    assert "200 of 440" in said and "240 slots" in said
