"""The serving loop over the paged 8-bit cache, with every code of every step checked: the slots that a step wrote against the exact
numbers, half a step of a code and the rotation's error (with fp32 tables: each entry is off by 4.4 * 2^-24, a channel by that of its
pair, sqrt(2) of the largest channel: 6.2 + 2 roundings of 2^-24, times sqrt(2), are 11.6 of the 18 that _check_append allows), and all
other slots bit for bit."""
import numpy as np
import pytest
import test_gpu_cache8 as base

from oracle import cache8 as o

pytestmark = pytest.mark.gpu


class _Loop(base._Loop):
    def check(self, step, q, out):
        cu, pos, _, k, v = step
        cos, sin = o.tables(pos, self.rot)
        before = self.codes
        want = o.append(before, self.scales, k, v, cu, self.table, self.lengths, cos, sin, self.layout)
        got = self.cache.pages.cpu().numpy(), base._np(self.cache.scales)
        case = cu, self.table, self.lengths, before, self.scales, k, v, cos, sin
        base._check_append(*got, want, before, case)
        new = sum(int(n) for n in np.diff(cu)) * self.heads * 2 * self.hd
        assert len(want[2]) * self.hd == new  # every token of the step was looked at
        self.codes, self.scales = got
        base._check_attention(base._np(out), o.attend(*got, base._np(q), cu, self.table, self.lengths, self.hd**-0.5, 150, 2), self.dtype,
                              self.hd, int(self.lengths.max()), None)


@pytest.mark.parametrize("dtype,layout,rot,hd", [("bf16", o.ADJACENT, 128, 128), ("fp16", o.HALVES, 64, 128), ("fp32", o.HALVES, 128, 128),
                                                 ("bf16", o.HALVES, 64, 64), ("fp16", o.ADJACENT, 256, 256)])
def test_every_code_of_a_serving_loop(gpu_device, dtype, layout, rot, hd):
    loop = _Loop(90, dtype=dtype, layout=layout, rot=rot, hd=hd)
    for news in ([100, 63, 1], [1, 1, 1], [1, 0, 1], [2, 3, 1], [150, 1, 40], [1, 1, 1]):
        step = loop.inputs(news)
        q, out = loop.run(loop.device(step))
        loop.check(step, q, out)


def test_every_code_of_replayed_steps(gpu_device):
    """A captured decoding step, replayed with other tokens and lengths, with eager work between the replays."""
    torch = base._t()
    loop = _Loop(91, dtype="bf16")
    step = loop.inputs([60, 127, 5])
    loop.check(step, *loop.run(loop.device(step)))
    step = loop.inputs([1, 1, 1])
    d = loop.device(step)
    ws = torch.empty(loop.cache.workspace_bytes(d["q"], 3), dtype=torch.uint8, device="cuda")
    loop.check(step, *loop.run(d, workspace=ws))
    pages, scales = loop.cache.pages.clone(), loop.cache.scales.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        q, out = loop.run(d, workspace=ws)
    loop.cache.pages.copy_(pages)
    loop.cache.scales.copy_(scales)
    for _ in range(6):
        step = loop.inputs([1, 1, 1])
        for name, x in loop.device(step).items():
            d[name].copy_(x)
        g.replay()
        loop.check(step, q, out)


def test_every_code_of_steps_on_two_streams(gpu_device):
    torch = base._t()
    loops = [_Loop(92), _Loop(93, dtype="fp32")]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for news in ([200, 3, 64], [1, 1, 1], [1, 0, 2]):
        todo = []
        for loop, s in zip(loops, streams):
            step = loop.inputs(news)
            d = loop.device(step)
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                torch.cuda._sleep(2_000_000)
                q, out = loop.run(d)
            todo.append((loop, step, q, out, d))
        for s in streams:
            s.synchronize()
        for loop, step, q, out, _ in todo:
            loop.check(step, q, out)
