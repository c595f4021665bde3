"""The serving example against a dense fp64 consumer that never quantises or pages anything."""
import math

import pytest
import torch

from examples import serve_prefix as E
from oracle import serving_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def served():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    return E.serve()


def _turn(x, first):
    """Rows of one request rotated from position ``first`` on, by complex numbers."""
    half = E.HEAD_DIM // 2
    w = torch.from_numpy(O.frequencies(E.HEAD_DIM, E.THETA))
    pos = torch.arange(first, first + x.shape[0], dtype=torch.float64)
    turn = torch.polar(torch.ones(1, dtype=torch.float64), pos[:, None] * w)[:, None]
    z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * turn
    return torch.cat([z.real, z.imag], -1)


def _dense(served):
    """Every request's hidden states of its prompt and generated tokens, in fp64."""
    f = lambda t: t.double().cpu()  # noqa: E731
    group = E.HEADS // E.KV_HEADS
    prompts, steps = [], []
    a = p = 0
    for n, m in zip(E.PREFIX, E.PROMPT):
        keys = [f(k[a:a + n]).view(n, E.KV_HEADS, E.HEAD_DIM) for k in served["dense"][0]]
        values = [f(v[a:a + n]).view(n, E.KV_HEADS, E.HEAD_DIM) for v in served["dense"][1]]

        def forward(x, pos):
            for l in range(E.LAYERS):
                t = x.shape[0]
                qkv = (x @ f(served["w_qkv"][l]).T).view(t, -1, E.HEAD_DIM)
                q = _turn(qkv[:, :E.HEADS], pos)
                keys[l] = torch.cat([keys[l], _turn(qkv[:, E.HEADS:E.HEADS + E.KV_HEADS], pos)])
                values[l] = torch.cat([values[l], qkv[:, E.HEADS + E.KV_HEADS:]])
                s = torch.einsum("thd,jhd->htj", q, keys[l].repeat_interleave(group, 1)) / math.sqrt(E.HEAD_DIM)
                late = torch.arange(keys[l].shape[0]) > torch.arange(pos, pos + t)[:, None]
                o = torch.einsum("htj,jhd->thd", torch.softmax(s.masked_fill(late, -math.inf), 2),
                                 values[l].repeat_interleave(group, 1))
                x = x + o.reshape(t, -1) @ f(served["w_out"][l]).T
                x = x * torch.rsqrt(x.square().mean(1, keepdim=True))
            return x

        x = forward(f(served["prompt_in"][p:p + m]), n)
        prompts.append(x)
        x = x[-1:]
        mine = []
        for i in range(E.STEPS):
            x = forward(x, n + m + i)
            mine.append(x)
        steps.append(torch.cat(mine))
        a, p = a + n, p + m
    return torch.cat(prompts), torch.stack(steps, 1)


def test_served_states_match_a_dense_consumer(served):
    """bf16 states (2^-9 each rounding, a dozen of them a layer) and 8-bit rows (a step of 1/127 of a page's
    largest value, about 1/32 of the typical one, in keys and values): together some percent of the states'
    size, which is 1.  A wrong page, position, mask or head would make states unrelated: a difference of 1.4."""
    prompts, steps = _dense(served)
    assert float((served["prompt_out"].double().cpu() - prompts).square().mean().sqrt()) < 0.1
    off = (served["tokens"].double().cpu() - steps).square().mean(2).sqrt()
    assert float(off.max()) < 0.4 and float(off.mean()) < 0.2


def test_the_cache_reads_back_as_it_was_filled(served):
    """The first layer's prefix rows, up to half a step of their page's scale and the bf16 rounding."""
    a = at = 0
    for n, h in zip(E.PREFIX, served["held"]):
        for x, y in zip((served["dense"][0][0], served["dense"][1][0]), served["back"]):
            x, y = x[a:a + n].float().view(n, E.KV_HEADS, E.HEAD_DIM), y[at:at + n].float()
            # pages that new tokens share may have grown: their scale is that of a few times the size
            assert float((x - y).abs().max()) <= 1.5 * float(x.abs().max()) / 127 + float(x.abs().max()) / 256
        a, at = a + n, at + h
