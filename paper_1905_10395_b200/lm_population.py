"""A population of small language models trained through the C ABI: an example of the operators in `lm` next to the leader step.

P workers, each a row of one parameter matrix x[P][ld].  A worker embeds its tokens, passes them through L blocks
    h = norm(x) w_pre,   u = relu([h_t, h_(t-1)] W1^T + b1),   y = u W2^T,   x <- x + sigmoid(gate) norm(y) w_post
and predicts the next token with the embedding table itself.  mixer="scan": a block sees all tokens before,
    h = norm(x) w_pre,   (v, z) = h W_in^T,   v = silu(conv(v)),   (dt, B, C) = v W_x^T,   y = scan(v, dt, B, C, z) W_out^T
with a short convolution and a selective state space scan (CausalConv, SelectiveScan) along the worker's T tokens.  One step is
    Embedding.forward, BlockNorm.forward at every block boundary, the products on the tensor cores (lsgd_bgemm_bf16), the loss,
    the same backwards, the table's gradient of the lookup added to that of the output layer (Embedding, accumulate),
    one AdamW launch over all tensors of all workers, which also rewrites the bf16 copies that the products read;
optimizer="ortho": the blocks' matrices are moved along their orthogonalised momentum instead (Orthogonalize);
every tau steps the workers' losses elect the leaders and lsgd_step pulls every worker towards its own (gradient zero, so the
update is the two pulls alone)."""
from __future__ import annotations

from contextlib import contextmanager
from typing import List, Optional, Tuple

import numpy as np
import torch

from . import api, lm


STATES, TAPS = 16, 4          # of a channel of the scan; of the convolution


def layout(V: int, D: int, F: int, L: int, mixer: str = "shift") -> Tuple[List[Tuple[str, tuple, int, bool]], int]:
    """(name, shape, offset, decayed) of a worker's tensors, each begun at a multiple of 32 floats, and the row length."""
    shapes = [("table", (V, D), True)]
    for i in range(L):
        shapes += [(f"w_pre{i}", (D,), False)]
        if mixer == "scan":
            shapes += [(f"w_in{i}", (2 * F, D), True), (f"taps{i}", (F, TAPS), False), (f"b_taps{i}", (F,), False),
                       (f"w_x{i}", (F + 2 * STATES, F), True), (f"a_log{i}", (F, STATES), False), (f"skip{i}", (F,), False),
                       (f"dt_bias{i}", (F,), False), (f"w_out{i}", (D, F), True)]
        else:
            shapes += [(f"w1_{i}", (F, 2 * D), True), (f"b1_{i}", (F,), False), (f"w2_{i}", (D, F), True)]
        shapes += [(f"w_post{i}", (D,), False), (f"gate{i}", (D,), False)]
    shapes.append((f"w_pre{L}", (D,), False))
    segs, at = [], 0
    for name, shape, decayed in shapes:
        segs.append((name, shape, at, decayed))
        at += (int(np.prod(shape)) + 31) // 32 * 32
    return segs, at


class LmPopulation:
    def __init__(self, P: int, G: int, *, V: int = 256, D: int = 64, F: int = 128, L: int = 2, T: int = 256, lr: float = 1e-2,
                 tau: int = 4, pull: float = 0.1, state: str = "8bit", seed: int = 0, device: str = "cuda:0", mixer: str = "shift",
                 optimizer: str = "adamw", lr_ortho: float = 2e-2):
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required (there is no CPU path)")
        if V % 8 or D % 8 or F % 8:
            raise ValueError("V, D and F are multiples of 8 (operands of the tensor-core products)")
        if mixer not in ("shift", "scan") or optimizer not in ("adamw", "ortho"):
            raise ValueError("mixer: shift or scan; optimizer: adamw or ortho")
        self.mixer, self.optimizer, self.lr_ortho = mixer, optimizer, lr_ortho
        self.P, self.V, self.D, self.F, self.L, self.T, self.lr, self.tau = P, V, D, F, L, T, lr, tau
        dev = torch.device(device)
        torch.cuda.set_device(dev)
        self.stream = torch.cuda.current_stream(dev)      # of all work, whatever stream is current at a call
        self.segs, self.ld = layout(V, D, F, L, mixer)
        gen = torch.Generator().manual_seed(seed)
        x = torch.zeros(P, self.ld)
        for name, shape, at, decayed in self.segs:
            n = int(np.prod(shape))
            if decayed:
                x[:, at:at + n] = torch.randn(P, n, generator=gen) * (0.02 if name == "table" else shape[1] ** -0.5)
            elif name.startswith("w_") or name.startswith("skip"):
                x[:, at:at + n] = 1.0
            elif name.startswith("taps"):
                x[:, at:at + n] = torch.randn(P, n, generator=gen) * TAPS ** -0.5
            elif name.startswith("a_log"):       # decays of 1 to N
                x[:, at:at + n] = torch.log(torch.arange(1, STATES + 1, dtype=torch.float32)).repeat(shape[0])
            elif name.startswith("dt_bias"):     # time steps of 0.001 to 0.1: the inverse of softplus
                step = torch.exp(torch.rand(P, n, generator=gen) * np.log(100.0) + np.log(1e-3))
                x[:, at:at + n] = step + torch.log(-torch.expm1(-step))
        self.x = x.to(dev)
        self.g = torch.zeros_like(self.x)
        self.zero = torch.zeros_like(self.x)
        self.copy = self.x.to(torch.bfloat16)
        view = lambda buf, name: self._view(buf, name)  # noqa: E731
        bf, f32 = dict(dtype=torch.bfloat16, device=dev), dict(dtype=torch.float32, device=dev)
        rows = lambda n, kind: torch.empty((P, T, n), **kind)  # noqa: E731

        # activations: the residual stream in fp32, what the products read in bf16
        self.tokens = torch.zeros((P, T), dtype=torch.int32, device=dev)
        self.target = torch.zeros((P, T), dtype=torch.int64, device=dev)
        self.res = [rows(D, f32) for _ in range(L + 1)]
        self.d_res = [rows(D, f32) for _ in range(L + 1)]
        self.h, self.d_h = [rows(D, bf) for _ in range(L + 1)], [rows(D, bf) for _ in range(L + 1)]
        if mixer == "scan":
            self._make_scan(rows, bf, view)
        else:
            self.cat, self.d_cat = [rows(2 * D, bf) for _ in range(L)], rows(2 * D, bf)
            self.u, self.d_u = [rows(F, bf) for _ in range(L)], rows(F, bf)
        self.y, self.d_y = [rows(D, bf) for _ in range(L)], [rows(D, bf) for _ in range(L)]
        self.logits = rows(V, f32)

        scale = float(D) ** 0.5
        self.embed = lm.Embedding(self.tokens, table=view(self.x, "table"), out=self.res[0], d_out=self.d_res[0],
                                  d_table=view(self.g, "table"), scale=scale, accumulate=True)
        # boundary 0 normalises the embedded tokens; boundary i + 1 closes block i and opens the next
        self.boundary = [lm.BlockNorm(x=self.res[0], h=self.h[0], out=self.res[0], w_pre=view(self.x, "w_pre0"),
                                      d_out=self.d_res[0] if L else None,
                                      d_h=self.d_h[0], dx=self.d_res[0], dw_pre=view(self.g, "w_pre0"))]
        for i in range(L):
            last = i + 1 == L
            self.boundary.append(lm.BlockNorm(
                x=self.res[i], y=self.y[i], gate=view(self.x, f"gate{i}"), w_post=view(self.x, f"w_post{i}"),
                w_pre=view(self.x, f"w_pre{i + 1}"), out=self.res[i + 1], h=self.h[i + 1], gate_act="sigmoid",
                d_out=None if last else self.d_res[i + 1], d_h=self.d_h[i + 1], dx=self.d_res[i], dy=self.d_y[i],
                d_gate=view(self.g, f"gate{i}"), dw_post=view(self.g, f"w_post{i}"), dw_pre=view(self.g, f"w_pre{i + 1}")))
        # the blocks' matrices, where they have an optimiser of their own: their update has a root mean square of about 0.2
        self.ortho = []
        if optimizer == "ortho":
            self.momentum = torch.zeros_like(self.x)
            for name, shape, _, decayed in self.segs:
                if decayed and name != "table":
                    out = torch.zeros((P, *shape), **bf)
                    op = lm.Orthogonalize(view(self.g, name), out, momentum=view(self.momentum, name), scale=0.2 * max(shape) ** 0.5)
                    self.ortho.append((op, out, view(self.x, name), view(self.copy, name)))
        adamw = [s for s in self.segs if not (self.ortho and s[3] and s[0] != "table")]
        pieces = lambda buf: [buf[p, at:at + int(np.prod(s))] for p in range(P) for _, s, at, _ in adamw]  # noqa: E731
        self.opt = lm.AdamW(pieces(self.x), pieces(self.g), copies=pieces(self.copy), state=state, beta2=0.95, seed=seed,
                            weight_decay=[0.1 if d else 0.0 for _ in range(P) for _, _, _, d in adamw])
        group_of = np.arange(P) * G // P
        cfg, keep = api.make_config(P=P, G=G, group_of=group_of, d=self.ld, ld=self.ld, eta=1.0, lambda_l=pull, lambda_g=pull / 2, tau=1,
                                    objective=api.OBJ_EXTERNAL, x=self.x, g=self.zero, stream=self.stream.cuda_stream)
        self.lsgd = api.Lsgd(cfg, keep)
        self.t = 0

    def _make_scan(self, rows, bf, view) -> None:
        """The activations of the scan's blocks and the operators on them: v and z are halves of one product's rows, dt, B and C parts of
        another's."""
        F, N, L = self.F, STATES, self.L
        self.vz, self.d_vz = [rows(2 * F, bf) for _ in range(L)], rows(2 * F, bf)
        self.v, self.d_v, self.d_v_x = [rows(F, bf) for _ in range(L)], rows(F, bf), rows(F, bf)
        self.dbc, self.d_dbc = [rows(F + 2 * N, bf) for _ in range(L)], rows(F + 2 * N, bf)
        self.u, self.d_u = [rows(F, bf) for _ in range(L)], rows(F, bf)
        self.conv, self.scan = [], []
        X, G = lambda n: view(self.x, n), lambda n: view(self.g, n)  # noqa: E731
        for i in range(L):
            vz, dbc, d_vz, d_dbc = self.vz[i], self.dbc[i], self.d_vz, self.d_dbc
            self.conv.append(lm.CausalConv(vz[..., :F], X(f"taps{i}"), bias=X(f"b_taps{i}"), out=self.v[i], d_out=self.d_v,
                                           dx=d_vz[..., :F], dw=G(f"taps{i}"), d_bias=G(f"b_taps{i}")))
            self.scan.append(lm.SelectiveScan(
                self.v[i], dbc[..., :F], X(f"a_log{i}"), dbc[..., F:F + N], dbc[..., F + N:], z=vz[..., F:], skip=X(f"skip{i}"),
                dt_bias=X(f"dt_bias{i}"), out=self.u[i], d_out=self.d_u, d_x=self.d_v_x, d_dt=d_dbc[..., :F], d_b=d_dbc[..., F:F + N],
                d_c=d_dbc[..., F + N:], d_z=d_vz[..., F:], d_a_log=G(f"a_log{i}"), d_skip=G(f"skip{i}"),
                d_dt_bias=G(f"dt_bias{i}")))

    def _view(self, buf: torch.Tensor, name: str) -> torch.Tensor:
        _, shape, at, _ = next(s for s in self.segs if s[0] == name)
        inner = [int(np.prod(shape[i + 1:])) for i in range(len(shape))]
        return torch.as_strided(buf, (self.P, *shape), (self.ld, *inner), buf.storage_offset() + at)

    def _product(self, a, b, c, *, a_t=False, b_t=False, epilogue: int, bias: Optional[torch.Tensor] = None,
                 mask: Optional[torch.Tensor] = None) -> None:
        """c[p] = a[p] b[p]^T with operands [P, rows, K]; a_t / b_t: stored [P, K, rows]."""
        d = api.BgemmDesc()
        d.a, d.b, d.c = a.data_ptr(), b.data_ptr(), c.data_ptr()
        d.M, d.N, d.K, d.batch = c.shape[1], c.shape[2], a.shape[1] if a_t else a.shape[2], self.P
        d.a_mn_major, d.b_mn_major = int(a_t), int(b_t)
        d.lda, d.ldb, d.ldc = a.stride(1), b.stride(1), c.stride(1)
        d.stride_a, d.stride_b, d.stride_c = a.stride(0), b.stride(0), c.stride(0)
        d.epilogue = epilogue
        if bias is not None:
            d.bias, d.stride_bias = bias.data_ptr(), bias.stride(0)
        if mask is not None:
            d.mask, d.ld_mask, d.stride_mask = mask.data_ptr(), mask.stride(1), mask.stride(0)
        api.lsgd_bgemm_bf16(d, self.stream.cuda_stream)

    @contextmanager
    def _in_order(self, *inputs: torch.Tensor):
        """The population's stream as the current one, behind the caller's and with the caller's behind it."""
        caller = torch.cuda.current_stream(self.x.device)
        if caller == self.stream:
            yield
            return
        self.stream.wait_stream(caller)
        for t in inputs:
            if t.is_cuda:
                t.record_stream(self.stream)
        with torch.cuda.stream(self.stream):
            yield
        caller.wait_stream(self.stream)

    def forward(self, tokens: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        """Mean next-token loss of every worker, [P]."""
        caller = torch.cuda.current_stream(self.x.device)
        with self._in_order(tokens, target):
            loss = self._forward(tokens, target)
        loss.record_stream(caller)
        return loss

    def _forward(self, tokens: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        D, W, X = self.D, lambda n: self._view(self.copy, n), lambda n: self._view(self.x, n)
        self.tokens.copy_(tokens)
        self.target.copy_(target)
        self.embed.forward()
        self.boundary[0].forward()
        for i in range(self.L):
            h = self.h[i]
            if self.mixer == "scan":
                self._product(h, W(f"w_in{i}"), self.vz[i], epilogue=3)
                self.conv[i].forward()
                self._product(self.v[i], W(f"w_x{i}"), self.dbc[i], epilogue=3)
                self.scan[i].forward()
                self._product(self.u[i], W(f"w_out{i}"), self.y[i], epilogue=3)
            else:
                cat = self.cat[i]
                cat[..., :D] = h
                cat[:, 1:, D:] = h[:, :-1]
                cat[:, 0, D:] = 0
                self._product(cat, W(f"w1_{i}"), self.u[i], epilogue=1, bias=X(f"b1_{i}"))
                self._product(self.u[i], W(f"w2_{i}"), self.y[i], epilogue=3)
            self.boundary[i + 1].forward()
        self._product(self.h[self.L], W("table"), self.logits, epilogue=0)
        self.logp = torch.log_softmax(self.logits, -1)
        return -self.logp.gather(2, self.target[..., None])[..., 0].mean(1)

    def backward(self) -> None:
        """Gradients of every worker's loss into g."""
        with self._in_order():
            self._backward()

    def _backward(self) -> None:
        D, W, Gv = self.D, lambda n: self._view(self.copy, n), lambda n: self._view(self.g, n)
        d_logits = self.logp.exp()
        d_logits.scatter_add_(2, self.target[..., None], torch.full_like(self.target[..., None], -1, dtype=torch.float32))
        d_logits = (d_logits / self.T).to(torch.bfloat16)
        self._product(d_logits, W("table"), self.d_h[self.L], b_t=True, epilogue=3)
        self._product(d_logits, self.h[self.L], Gv("table"), a_t=True, b_t=True, epilogue=0)
        for i in reversed(range(self.L)):
            self.boundary[i + 1].backward()
            if self.mixer == "scan":
                self._scan_backward(i, W, Gv)
                continue
            self._product(self.d_y[i], W(f"w2_{i}"), self.d_u, b_t=True, epilogue=2, mask=self.u[i])
            self._product(self.d_y[i], self.u[i], Gv(f"w2_{i}"), a_t=True, b_t=True, epilogue=0)
            self._product(self.d_u, self.cat[i], Gv(f"w1_{i}"), a_t=True, b_t=True, epilogue=0)
            Gv(f"b1_{i}").copy_(self.d_u.float().sum(1))
            self._product(self.d_u, W(f"w1_{i}"), self.d_cat, b_t=True, epilogue=3)
            d_h = self.d_cat[..., :D].float()
            d_h[:, :-1] += self.d_cat[:, 1:, D:].float()
            self.d_h[i].copy_(d_h)
        self.boundary[0].backward()
        self.embed.backward()

    def _scan_backward(self, i: int, W, Gv) -> None:
        self._product(self.d_y[i], W(f"w_out{i}"), self.d_u, b_t=True, epilogue=3)
        self._product(self.d_y[i], self.u[i], Gv(f"w_out{i}"), a_t=True, b_t=True, epilogue=0)
        self.scan[i].backward()
        self._product(self.d_dbc, self.v[i], Gv(f"w_x{i}"), a_t=True, b_t=True, epilogue=0)
        self._product(self.d_dbc, W(f"w_x{i}"), self.d_v, b_t=True, epilogue=3)
        self.d_v.add_(self.d_v_x)
        self.conv[i].backward()
        self._product(self.d_vz, self.h[i], Gv(f"w_in{i}"), a_t=True, b_t=True, epilogue=0)
        self._product(self.d_vz, W(f"w_in{i}"), self.d_h[i], b_t=True, epilogue=3)

    def step(self, tokens: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        loss = self.forward(tokens, target)
        with self._in_order():
            self._backward()
            self.opt.step(self.lr)
            for op, out, x, copy in self.ortho:
                op.forward()
                x.mul_(1.0 - self.lr_ortho * 0.1).add_(out, alpha=-self.lr_ortho)
                copy.copy_(x)
            self.t += 1
            if self.t % self.tau == 0:
                if self.ortho:
                    self.ortho[0][0].check()     # one status word of them all: no leader is followed from a failed update
                self.lsgd.elect(loss)
                self.lsgd.step()
                self.copy.copy_(self.x)          # the pulls moved the parameters: the products' copies follow
        return loss

    def close(self) -> None:
        self.lsgd.destroy()
        self.opt.destroy()


def markov_tokens(P: int, T: int, V: int, gen: torch.Generator) -> Tuple[torch.Tensor, torch.Tensor]:
    """Sequences in which a token is followed by one of two fixed ones: (tokens, next tokens), [P, T] each."""
    tok = torch.empty((P, T + 1), dtype=torch.int64)
    tok[:, 0] = torch.randint(0, V, (P,), generator=gen)
    coin = torch.randint(0, 2, (P, T), generator=gen)
    for t in range(T):
        tok[:, t + 1] = (tok[:, t] * 5 + 7 + 31 * coin[:, t]) % V
    return tok[:, :-1].contiguous(), tok[:, 1:].contiguous()


def main(steps: int = 200) -> None:
    pop = LmPopulation(8, 2)
    gen = torch.Generator().manual_seed(1)
    for t in range(steps):
        tok, target = markov_tokens(pop.P, pop.T, pop.V, gen)
        loss = pop.step(tok.cuda(), target.cuda())
        if t % 20 == 0 or t + 1 == steps:
            print(f"step {t}: loss of the best worker {loss.min().item():.3f}, of all {loss.mean().item():.3f} (the source's entropy is 0.693)")
    pop.close()


if __name__ == "__main__":
    main()
