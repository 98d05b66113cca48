"""Text generation as a side task: a batch of sequences behind one shared prompt, a token each a step, in a stage's bubbles.

A small decoder (random weights) on the library's own operators: fr_gemm_bf16 for the products, fr_kv_append (positions rotated,
keys and values into pages), fr_attend_shared (the prompt's keys lie there once for the whole batch), fr_sample (the next token);
torch does the rest (norms, residual sums, table look-ups).  A step is one token of every sequence: short, of known length, and
the state between two steps lies in device memory, so a bubble takes as many steps as fit and the next bubble goes on from there.
A step is captured in a HIP graph once; run_step replays it on the side stream.

    python examples/generate_in_bubbles.py            # a 1F1B stage with timed operations, tokens generated in its bubbles
"""
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2409_06941_amd as fr


class Decoder:
    """Pre-norm decoder with grouped heads.  Batch, widths and vocabulary are multiples of 256 (fr_gemm_bf16)."""

    def __init__(self, batch=256, prompt=512, new=32, layers=2, hidden=512, q_heads=8, kv_heads=2, head_dim=64, ffn=1024,
                 vocab=4096, page=16, temperature=0.8, top_k=50, top_p=0.95, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        weight = lambda n, k: (torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).to(torch.bfloat16)
        self.batch, self.prompt_len, self.new = batch, prompt, new
        self.hidden, self.q_heads, self.kv_heads, self.head_dim, self.page = hidden, q_heads, kv_heads, head_dim, page
        self.qkv_heads = q_heads + 2 * kv_heads
        self.layers = [dict(qkv=weight(self.qkv_heads * head_dim, hidden), out=weight(hidden, q_heads * head_dim),
                            up=weight(ffn, hidden), down=weight(hidden, ffn)) for _ in range(layers)]
        self.embed, self.unembed = weight(vocab, hidden), weight(vocab, hidden)
        # pages: the prompt's first, then every sequence's own
        self.own_pages = -(-new // page)
        prompt_pages = -(-prompt // page)
        pages = prompt_pages + batch * self.own_pages
        cache = lambda: torch.zeros((pages, kv_heads, page, head_dim), dtype=torch.bfloat16, device="cuda")
        self.caches = [fr.KvPages(cache(), cache()) for _ in range(layers)]
        self.prefix_pages = torch.arange(prompt_pages, dtype=torch.int32, device="cuda")
        self.pages = torch.arange(prompt_pages, pages, dtype=torch.int32, device="cuda").view(batch, self.own_pages)
        inv = 10000.0 ** (-torch.arange(0, head_dim, 2, dtype=torch.float64, device="cuda") / head_dim)
        angle = torch.arange(prompt + new, dtype=torch.float64, device="cuda")[:, None] * inv
        self.rotary = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        # what a step reads and moves on: how many tokens there are, the random numbers of every step, the tokens
        self.done = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.uniform = torch.rand((new, batch), generator=g, device="cuda")
        self.first = torch.randint(0, vocab, (batch,), generator=g, device="cuda")
        self.prompt = torch.randint(0, vocab, (prompt,), generator=g, device="cuda")
        self.tokens = torch.zeros((new, batch), dtype=torch.int32, device="cuda")
        self.current = torch.zeros(batch, dtype=torch.int64, device="cuda")
        full = lambda x, dtype: torch.full((batch,), x, dtype=dtype, device="cuda")
        self.settings = dict(temperature=full(temperature, torch.float32), top_k=full(top_k, torch.int32), top_p=full(top_p, torch.float32))
        self.limits = dict(prefix_len=prompt, max_own_len=new)
        self.rows = torch.arange(batch, device="cuda")
        q = torch.empty((batch, q_heads, head_dim), dtype=torch.bfloat16, device="cuda")
        attend = max(fr.fr_attend_shared_workspace_bytes(c, q, batch, **self.limits) for c in self.caches)
        choose = fr.fr_sample_workspace_bytes(torch.empty((batch, vocab), dtype=torch.bfloat16, device="cuda"))
        self.workspace = torch.empty(max(attend, choose, 1), dtype=torch.uint8, device="cuda")
        self.logits = None
        self.graph = None

    @staticmethod
    def _norm(x):
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5)).to(torch.bfloat16)

    @staticmethod
    def _product(x, weight, stream):
        y = torch.empty((x.shape[0], weight.shape[0]), dtype=torch.bfloat16, device="cuda")
        fr.fr_gemm_bf16(x, weight, y, x.shape[0], weight.shape[0], weight.shape[1], stream)
        return y

    def _forward(self, tokens, slot, position, attend, stream):
        """Hidden states of these tokens; `attend(cache, q, out)` reads the cache that they have been appended to."""
        x = self.embed[tokens].float()
        n, q_width = tokens.shape[0], self.q_heads * self.head_dim
        for layer, cache in zip(self.layers, self.caches):
            qkv = self._product(self._norm(x), layer["qkv"], stream).view(n, self.qkv_heads, self.head_dim)
            q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
            out = torch.empty((n, self.q_heads, self.head_dim), dtype=torch.bfloat16, device="cuda")
            fr.fr_kv_append(cache, k, v, slot, q=q, q_out=q, position=position, rotary=self.rotary, stream=stream)
            attend(cache, q, out)
            x = x + self._product(out.view(n, q_width), layer["out"], stream).float()
            up = self._product(self._norm(x), layer["up"], stream)
            x = x + self._product(torch.nn.functional.gelu(up.float()).to(torch.bfloat16), layer["down"], stream).float()
        return x

    def prefill(self):
        """Keys and values of the prompt, once for every sequence: as one sequence with own keys only."""
        stream, n = torch.cuda.current_stream(), self.prompt_len
        position = torch.arange(n, dtype=torch.int32, device="cuda")
        length = torch.full((1,), n, dtype=torch.int32, device="cuda")
        begin = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        limits = dict(prefix_len=0, max_own_len=n, max_q=n)
        q = torch.empty((n, self.q_heads, self.head_dim), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(1, fr.fr_attend_shared_workspace_bytes(self.caches[0], q, 1, **limits)), dtype=torch.uint8, device="cuda")
        attend = lambda cache, q, out: fr.fr_attend_shared(cache, q, out, self.prefix_pages.view(1, -1), length, self.head_dim ** -0.5,
                                                           q_begin=begin, workspace=ws, stream=stream, **limits)
        self._forward(self.prompt, position.long(), position, attend, stream)          # (the prompt's pages are the first)
        self.reset()

    def reset(self):
        self.done.zero_()
        self.tokens.zero_()
        self.current.copy_(self.first)

    def step(self):
        """One token of every sequence, on the current stream; where it stands is read from the device, so that it can be replayed."""
        stream = torch.cuda.current_stream()
        at = self.done.expand(self.batch)
        slot = self.pages[self.rows, at // self.page].long() * self.page + at % self.page
        position, length = (at + self.prompt_len).int(), (at + 1).int()
        attend = lambda cache, q, out: fr.fr_attend_shared(cache, q, out, self.pages, length, self.head_dim ** -0.5,
                                                           prefix_pages=self.prefix_pages, workspace=self.workspace, stream=stream, **self.limits)
        x = self._forward(self.current, slot, position, attend, stream)
        self.logits = self._product(self._norm(x), self.unembed, stream)
        token = torch.empty(self.batch, dtype=torch.int32, device="cuda")
        fr.fr_sample(self.logits, self.uniform.index_select(0, self.done)[0].contiguous(), token, workspace=self.workspace, stream=stream,
                     **self.settings)
        self.tokens.index_copy_(0, self.done, token[None])
        self.current.copy_(token)
        self.done.add_(1)

    def capture(self):
        """The step as a graph; the first token is generated on the way and forgotten again."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step()
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.step()
        self.reset()
        torch.cuda.synchronize()


class GenerationTask:
    """fr_task_ops over a captured Decoder: one run = `new` tokens of every sequence, a segment = a tile = one token."""

    def __init__(self, model, step_ns, bytes_used):
        self.model, self.step_ns, self.at = model, int(step_ns), 0
        b = fr.binding
        self.bytes = bytes_used
        self.ops = fr.fr_task_ops(b.CREATE_FN(lambda user: 0), b.INIT_FN(self._init), b.PLAN_FN(self._plan), b.RUN_FN(self._run),
                                  b.STOP_FN(lambda user: 0))
        self.profile = fr.fr_task_profile(bytes_used + (1 << 20), self.step_ns)

    def _init(self, user, alloc, stream):
        return fr.lib().fr_alloc_charge(alloc, self.bytes)          # (the tensors are torch's: booked, not taken)

    def _plan(self, user, budget_ns, launch_cost_ns, out):
        s = out.contents
        s.modelled_ns = s.work_units = 0
        s.run = s.cost_class = 0
        s.segment, s.tile0, s.tile1 = self.at, 0, 0
        s.finished, s.completes_run = int(self.at >= self.model.new), 0
        if not s.finished and self.step_ns + launch_cost_ns <= budget_ns:
            s.modelled_ns, s.work_units, s.tile1 = self.step_ns, self.model.batch, 1
            s.completes_run = int(self.at + 1 == self.model.new)
        return 0

    def _run(self, user, stream, planned):
        with torch.cuda.stream(torch.cuda.ExternalStream(stream)):
            self.model.graph.replay()
        self.at += 1
        return 0


def standalone(model):
    """All tokens outside any bubble; returns them and the time of a step, ns."""
    model.reset()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    model.graph.replay()
    model.reset()
    torch.cuda.synchronize()
    begin.record()
    for _ in range(model.new):
        model.graph.replay()
    end.record()
    torch.cuda.synchronize()
    return model.tokens.clone(), begin.elapsed_time(end) * 1e6 / model.new


def harvest(model, step_ns, epochs=8, f_ns=2_000_000, b_ns=4_000_000):
    """The same tokens in the bubbles of stage 2 of 4 (1F1B, 8 micro-batches, timed operations); returns tokens, progress, bubble time."""
    model.reset()
    torch.cuda.synchronize()
    ctx = fr.Context(device_id=0, guard_ns=200_000, launch_cost_ns=30_000, max_chunk_ns=2_000_000, mem_available_bytes=1 << 38)
    task = GenerationTask(model, 1.25 * step_ns + 20_000, sum(2 * c._keep[0].numel() * 2 for c in model.caches))
    tid = ctx.fr_task_register(task.ops, None, task.profile)
    load = fr.Load(fr.FR_LOAD_BUSYWAIT, fp_ns=f_ns, bp_ns=b_ns)
    stage = fr.Stage(fr.FR_SCHED_1F1B, 4, 8, 2, f_ns, b_ns, load, torch.cuda.Stream())
    bubble_ns = 0
    for _ in range(epochs):
        bubble_ns += stage.fr_stage_run_epoch(ctx).bubble_ns
        if task.at >= model.new:
            break
    progress = ctx.fr_query_progress(tid)
    ctx.fr_task_stop(tid)
    torch.cuda.synchronize()
    stage.fr_stage_destroy(), load.fr_load_destroy(), ctx.fr_destroy()
    return model.tokens.clone(), progress, bubble_ns


def main():
    model = Decoder(new=64)
    model.prefill()
    model.capture()
    want, step_ns = standalone(model)
    t = time.time()
    got, progress, bubble_ns = harvest(model, step_ns)
    print("a step of %d sequences behind %d tokens: %.0f us; %d of %d steps in the bubbles (%.1f ms of bubble time, %.2f s wall), "
          "%d overruns; tokens as outside of bubbles: %s" %
          (model.batch, model.prompt_len, step_ns / 1e3, progress.steps, model.new, bubble_ns / 1e6, time.time() - t, progress.overruns,
           torch.equal(got, want)))


if __name__ == "__main__":
    main()
