"""The MLP of a language model with experts, in 8-bit floating point: the layer of experts with its router and residual, a dense MLP beside it and a
dense layer, for a prompt and then token by token.

    python examples/expert_block.py [--tokens 512] [--steps 8] [--d 1024] [--ff 512] [--experts 16] [--top-k 2]

Weights are random bf16 matrices that the plans quantize; the outputs are compared with the same block in unquantized fp32 torch.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class ExpertBlock:
    """x -> y = x + experts(x), y -> y + mlp(y) (an MLP that all tokens share), then a dense layer: what decoder layers do between two attentions."""

    def __init__(self, d, ff, experts, top_k, seed=0):
        import torch

        import paper_2510_26771_amd as st
        g = torch.Generator(device="cuda").manual_seed(seed)

        def matrix(*shape):
            return (torch.randn(shape, device="cuda", generator=g) * shape[-1] ** -0.5).to(torch.bfloat16)
        self.st, self.d, self.experts, self.top_k = st, d, experts, top_k
        self.w_router = matrix(experts, d).float()
        self.w_up, self.w_down, self.w_dense = matrix(experts, 2, ff, d), matrix(experts, d, ff), matrix(d, d)
        self.w_shared_up, self.w_shared_down = matrix(ff, d), matrix(d, ff) * 0.5
        bf16 = st.STAMP_BF16
        self.up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=experts, gated=1, w_dtype=bf16), self.w_up)
        self.down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d, experts=experts, w_dtype=bf16), self.w_down)
        self.dense = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=d, w_dtype=bf16), self.w_dense)
        self.shared_up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, w_dtype=bf16), self.w_shared_up)
        self.shared_down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d, w_dtype=bf16), self.w_shared_down)
        self.room = {}

    def buffers(self, tokens):
        """Routing, workspaces and output for so many tokens: kept, as a serving loop would."""
        import torch
        if tokens not in self.room:
            st = self.st
            self.room[tokens] = (st.Routing(tokens, self.experts, self.top_k), st.moe_workspace(self.up, self.down, tokens, self.top_k),
                                 st.mlp_workspace(self.shared_up, self.shared_down, tokens), self.dense.alloc_workspace(tokens), *(torch.empty((tokens, self.d), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        return self.room[tokens]

    def __call__(self, x):
        st = self.st
        routing, ws, ws_mlp, ws_dense, y, out = self.buffers(x.shape[0])
        st.moe_forward(self.w_router, self.up, self.down, x, routing, y, ws, residual=x)
        st.mlp_forward(self.shared_up, self.shared_down, y, y, ws_mlp, "gelu", residual=y)
        self.dense.linear_forward(y, out, ws_dense)
        return out

    def reference(self, x):
        import torch
        x = x.float()
        top, ids = (x @ self.w_router.t()).topk(self.top_k, dim=1)
        weights = torch.softmax(top, 1)
        y = torch.zeros_like(x)
        for e in range(self.experts):
            t, j = torch.nonzero(ids == e, as_tuple=True)
            if t.numel():
                gate, up = (x[t] @ self.w_up[e, i].float().t() for i in (0, 1))
                y.index_add_(0, t, weights[t, j, None] * ((torch.nn.functional.silu(gate) * up) @ self.w_down[e].float().t()))
        y = x + y
        y = y + torch.nn.functional.gelu(y @ self.w_shared_up.float().t()) @ self.w_shared_down.float().t()
        return y @ self.w_dense.float().t()


def main(argv=None):
    import torch
    p = argparse.ArgumentParser()
    for name, value in (("tokens", 512), ("steps", 8), ("d", 1024), ("ff", 512), ("experts", 16), ("top-k", 2)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args(argv)
    block = ExpertBlock(a.d, a.ff, a.experts, a.top_k)
    x = torch.randn((a.tokens + a.steps, a.d), device="cuda").to(torch.bfloat16)
    parts = [x[: a.tokens]] + [x[a.tokens + i: a.tokens + i + 1] for i in range(a.steps)]
    out = torch.cat([block(part).clone() for part in parts]).float()
    want = block.reference(x)
    err = float((out - want).norm() / want.norm())
    alone = torch.cat([block(row[None]).clone() for row in x[: min(4, a.tokens)]]).float()
    apart = float((alone - out[: alone.shape[0]]).norm() / out[: alone.shape[0]].norm())
    print(f"prompt of {a.tokens} tokens and {a.steps} single tokens: {err:.3%} from the unquantized block, "
          f"single tokens {apart:.2e} from the same tokens of the prompt")
    return err, apart


if __name__ == "__main__":
    main()
