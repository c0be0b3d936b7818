"""Device buffers and launch sequence of one XNOR block per layer.

Marshalling only: it owns torch tensors and calls the C-ABI entry points in
the paper's order (weight binarisation, then BN -> BinActiv -> BinConv).
"""
import torch

from . import binding as B
from . import workloads as wl


class LayerBuffers:
    """All device tensors of one layer; inputs are filled by the caller."""

    def __init__(self, shape, device="cuda", with_acc=False, with_bn=True, variant="xnor", kbits=2):
        """variant: "xnor" (the block of Eq. 11), "bwn" (real inputs, binary weights, Eq. 1),
        "kbit" (q_k activations with `kbits` bits in place of sign) or "bgrad" (the layer's backward
        convolution with a binarised gradient: x is then the gradient at the layer's output,
        [N][C_out][H_out][W_out], and out the gradient at its input, [N][C_in][H][W])."""
        s = shape
        self.variant, self.kbits = variant, kbits
        self.shape = s
        self.desc = B.desc_of(s)
        self.x = torch.empty((s.N, s.C_in, s.H, s.W), dtype=torch.float32, device=device)
        self.w = torch.empty((s.C_out, s.C_in, s.k, s.k), dtype=torch.float32, device=device)
        self.bn_scale = torch.ones((s.C_in,), dtype=torch.float32, device=device) if with_bn else None
        self.bn_shift = torch.zeros((s.C_in,), dtype=torch.float32, device=device) if with_bn else None
        self.w_packed, self.alpha = B.alloc_weights(s.C_out, s.C_in, s.k, s.k, device)
        self.x_packed, self.A, self.K = B.alloc_binactiv(self.desc, device)
        self.out = B.alloc_out(self.desc, device=device)
        self.acc = B.alloc_out(self.desc, torch.int32, device) if with_acc else None
        self.residual = None
        if variant == "bwn":
            self.x_stream = B.alloc_bwn_input(self.desc, device)
        elif variant == "kbit":
            self.x_planes = torch.empty((kbits,) + tuple(self.x_packed.shape), dtype=torch.int32,
                                        device=device)
        elif variant == "bgrad":
            self.x = torch.empty(tuple(self.out.shape), dtype=torch.float32, device=device)
            self.wT_packed = B.alloc_weights_transposed(s.C_out, s.C_in, s.k, s.k, device)
            self.gmax, self.g_stream, self.out = B.alloc_bgrad(self.desc, device)

    def binarize_weights(self, stream=None):
        B.xnor_binarize_weights(self.w, self.w_packed, self.alpha, stream)
        if self.variant == "bgrad":
            B.xnor_binarize_weights_transposed(self.w, self.wT_packed, stream)

    def binactiv(self, stream=None):
        if self.variant == "bgrad":
            return                   # the gradient is scaled and laid out inside the backward call
        if self.variant == "bwn":
            B.xnor_bwn_prepare_input(self.x, self.bn_scale, self.bn_shift, self.desc, self.x_stream, stream)
        elif self.variant == "kbit":
            B.xnor_binactiv_kbit(self.x, self.bn_scale, self.bn_shift, self.desc, self.kbits,
                                 self.x_planes, self.A, self.K, stream)
        else:
            B.xnor_binactiv(self.x, self.bn_scale, self.bn_shift, self.desc, self.x_packed, self.A,
                            self.K, stream)

    def conv(self, stream=None):
        if self.variant == "bgrad":
            B.xnor_binary_gradient_backward(self.x, self.wT_packed, self.alpha, self.desc, self.gmax,
                                            self.g_stream, self.out, stream)
        elif self.variant == "bwn":
            B.xnor_bwn_conv2d_forward(self.x_stream, self.w_packed, self.alpha, self.residual,
                                      self.desc, self.out, stream)
        elif self.variant == "kbit":
            B.xnor_conv2d_forward_kbit(self.x_planes, self.kbits, self.w_packed, self.alpha, self.K,
                                       self.residual, self.desc, self.out, self.acc, stream)
        else:
            B.xnor_conv2d_forward(self.x_packed, self.w_packed, self.alpha, self.K, self.residual,
                                  self.desc, self.out, self.acc, stream)

    def forward(self, stream=None, with_weights=True):
        if with_weights:
            self.binarize_weights(stream)
        self.binactiv(stream)
        self.conv(stream)

    # algorithmic bytes, as the roofline of each kernel counts them
    def binactiv_launches(self):
        if self.variant == "bgrad":
            return 0
        if self.variant == "bwn":
            return 1
        if self.variant == "kbit":
            return B.xnor_binactiv_kbit_launches(self.desc, self.kbits, self.bn_scale is not None)
        return B.xnor_binactiv_launches(self.desc, self.bn_scale is not None)

    def launches(self):
        """Kernels one forward() launches: binarize 1, BinActiv 1 or 2 (pack + A, box filter; one
        kernel where a block streams whole images), BinConv 1 (k-bit: one per pass)."""
        if self.variant == "bgrad":
            return 2 + 3             # two weight packings; maximum, gradient stream, convolution
        conv = 1
        if self.variant == "kbit":
            conv = B.xnor_conv2d_plan(self.desc, self.kbits).launches
        return 1 + self.binactiv_launches() + conv

    def binactiv_bytes(self):
        if self.variant == "bgrad":
            return 0
        s = self.shape
        ho, wo = wl.out_hw(s)
        cw = (s.C_in + 31) // 32
        px = s.N * s.H * s.W
        # A is written once and, where K comes from a second kernel, read once
        a_passes = 2 if self.binactiv_launches() == 2 else 1
        return 4 * (px * s.C_in + px * cw + a_passes * px + s.N * ho * wo)

    def conv_bytes(self):
        s = self.shape
        ho, wo = wl.out_hw(s)
        cw = (s.C_in + 31) // 32
        m = s.N * ho * wo
        return 4 * (s.N * s.H * s.W * cw + s.C_out * s.k * s.k * cw + m + s.C_out + m * s.C_out)

    def weight_bytes(self):
        s = self.shape
        return 4 * s.C_out * s.C_in * s.k * s.k




class ChainRunner:
    """The 16 binary 3x3 layers of the ResNet-18 variant (Section 4.2) as 8 basic blocks:

        y1 = BinConv1(BinActiv(BN1(x)))
        y2 = BinConv2(BinActiv(BN2(y1))) + shortcut(x)

    shortcut = identity, or the fp32 1x1 stride-2 projection where the shape
    changes.  Launch sequence and buffers only; every step is a library call.
    BatchNorm enters as per-channel (scale, shift) vectors that the caller sets
    (see `calibrate`).
    """

    def __init__(self, N, device="cuda", keep_acc=False):
        self.N = N
        self.shapes = wl.chain_shapes(N)
        self.device = device
        s0 = self.shapes[0]
        self.x0 = torch.empty((N, s0.C_in, s0.H, s0.W), dtype=torch.float32, device=device)
        self.layers = []
        for s in self.shapes:
            d = B.desc_of(s)
            L = {"shape": s, "desc": d}
            L["w"] = torch.empty((s.C_out, s.C_in, s.k, s.k), dtype=torch.float32, device=device)
            L["w_packed"], L["alpha"] = B.alloc_weights(s.C_out, s.C_in, s.k, s.k, device)
            L["x_packed"], L["A"], L["K"] = B.alloc_binactiv(d, device)
            L["scale"] = torch.ones((s.C_in,), dtype=torch.float32, device=device)
            L["shift"] = torch.zeros((s.C_in,), dtype=torch.float32, device=device)
            L["out"] = B.alloc_out(d, device=device)
            L["acc"] = B.alloc_out(d, torch.int32, device) if keep_acc else None
            self.layers.append(L)
        # projection shortcuts: one per block whose first layer has stride 2
        self.proj = {}
        for i in range(0, len(self.shapes), 2):
            s = self.shapes[i]
            if s.stride != 1 or s.C_in != s.C_out:
                ho, wo = wl.out_hw(s)
                self.proj[i] = {
                    "w": torch.empty((s.C_out, s.C_in), dtype=torch.float32, device=device),
                    "out": torch.empty((N, s.C_out, ho, wo), dtype=torch.float32, device=device)}

    def layer_input(self, i):
        return self.x0 if i == 0 else self.layers[i - 1]["out"]

    def binarize_weights(self, stream=None):
        for L in self.layers:
            B.xnor_binarize_weights(L["w"], L["w_packed"], L["alpha"], stream)

    def run_layer(self, i, stream=None):
        """BN -> BinActiv -> BinConv of layer i (plus the block's shortcut on odd i)."""
        L = self.layers[i]
        x = self.layer_input(i)
        B.xnor_binactiv(x, L["scale"], L["shift"], L["desc"], L["x_packed"], L["A"], L["K"], stream)
        residual = None
        if i % 2 == 1:
            b0 = i - 1
            if b0 in self.proj:
                P = self.proj[b0]
                B.xnor_shortcut_conv1x1(self.layer_input(b0), P["w"], self.shapes[b0].stride,
                                        P["out"], stream)
                residual = P["out"]
            else:
                residual = self.layer_input(b0)
        B.xnor_conv2d_forward(L["x_packed"], L["w_packed"], L["alpha"], L["K"], residual,
                              L["desc"], L["out"], L["acc"], stream)
        return residual

    def forward(self, stream=None):
        for i in range(len(self.layers)):
            self.run_layer(i, stream)
        return self.layers[-1]["out"]

    def prepare_fused(self):
        """Buffers of the fused forward: for every layer but the last, the partial |y| planes
        its fused epilogue writes (0 parts: the shape is not covered and the layer runs the two
        plain calls).  The engine in force now must be the one used by forward_fused."""
        self.fused_parts = []
        for i, L in enumerate(self.layers[:-1]):
            parts = B.xnor_conv2d_binactiv_parts(L["desc"])
            self.fused_parts.append(parts)
            ho, wo = wl.out_hw(L["shape"])
            L["A_parts"] = torch.empty((max(parts, 1), self.N, ho, wo), dtype=torch.float32,
                                       device=self.device)
        self.fused_parts.append(0)

    def forward_fused(self, stream=None):
        """The same chain with each BinConv emitting the next layer's BinActiv from its epilogue.
        The output of a block's first convolution is consumed only by that BinActiv, so it is
        never written as fp32; a block's output is (it is the next block's shortcut input)."""
        n = len(self.layers)
        L0 = self.layers[0]
        B.xnor_binactiv(self.x0, L0["scale"], L0["shift"], L0["desc"], L0["x_packed"], L0["A"], L0["K"],
                        stream)
        for i, L in enumerate(self.layers):
            residual = None
            if i % 2 == 1:
                b0 = i - 1
                if b0 in self.proj:
                    P = self.proj[b0]
                    B.xnor_shortcut_conv1x1(self.layer_input(b0), P["w"], self.shapes[b0].stride,
                                            P["out"], stream)
                    residual = P["out"]
                else:
                    residual = self.layer_input(b0)
            parts = self.fused_parts[i]
            if parts > 0:
                nxt = self.layers[i + 1]
                out = L["out"] if i % 2 == 1 else None
                B.xnor_conv2d_forward_binactiv(L["x_packed"], L["w_packed"], L["alpha"], L["K"],
                                               residual, L["desc"], out, nxt["scale"], nxt["shift"],
                                               nxt["x_packed"], L["A_parts"], stream)
                B.xnor_binactiv_finish(L["A_parts"], parts, nxt["desc"], nxt["A"], nxt["K"], stream)
            else:
                B.xnor_conv2d_forward(L["x_packed"], L["w_packed"], L["alpha"], L["K"], residual,
                                      L["desc"], L["out"], None, stream)
                if i + 1 < n:
                    nxt = self.layers[i + 1]
                    B.xnor_binactiv(L["out"], nxt["scale"], nxt["shift"], nxt["desc"],
                                    nxt["x_packed"], nxt["A"], nxt["K"], stream)
        return self.layers[-1]["out"]

    def calibrate(self, eps=1e-5, stream=None):
        """Sets every BatchNorm to the statistics of its own input on the current batch
        (biased variance, gamma = 1, beta = 0), layer by layer.  Set-up, not the timed path:
        the statistics are plain torch reductions; the folded (scale, shift) vectors are what
        the library (and any checker) receives."""
        for i, L in enumerate(self.layers):
            x = self.layer_input(i).double()
            mean = x.mean(dim=(0, 2, 3))
            var = x.var(dim=(0, 2, 3), unbiased=False)
            scale = 1.0 / torch.sqrt(var + eps)
            L["scale"].copy_(scale.float())
            L["shift"].copy_((-mean * scale).float())
            self.run_layer(i, stream)

    def launches_per_forward(self):
        # per layer: BinActiv (one or two kernels), conv; plus one kernel per projection shortcut
        act = sum(B.xnor_binactiv_launches(L["desc"], True) for L in self.layers)
        return act + len(self.layers) + len(self.proj)

    def macs(self):
        return sum(wl.macs(s) for s in self.shapes)


class TokenBlock:
    """Buffers and calls of a projection in a decoder's layer: the residual's addition, the norm, and the product
    with 4-bit weights, on bfloat16 rows of tokens.

    quant: None (the product reads the norm in bfloat16), "i8" or "e4m3" (in 8 bits, one scale for each row),
    "i8_groups" or "e4m3_groups" (a scale for each of the weights' groups)."""

    def __init__(self, rows, K, N, group=128, zeros=False, quant=None, eps=1e-5, device="cuda"):
        if quant not in (None, "i8", "e4m3", "i8_groups", "e4m3_groups"):
            raise ValueError("quant: None, 'i8', 'e4m3', 'i8_groups' or 'e4m3_groups', not %r" % (quant,))
        if quant is not None and quant.endswith("_groups") and K % group:
            raise ValueError("scales of groups want K (%d) in whole groups of %d" % (K, group))
        bf16 = dict(dtype=torch.bfloat16, device=device)
        self.eps, self.d = eps, B.make_w4_desc(N, K, group)
        self.x, self.residual = torch.empty((rows, K), **bf16), torch.empty((rows, K), **bf16)
        self.weight = torch.ones((K,), dtype=torch.float32, device=device)
        self.packed, self.scales, self.zeros = B.alloc_w4(self.d, zeros, device)
        self.out = torch.empty((rows, N), **bf16)
        self.y = self.q = self.q_scales = None
        self.q_group = group if quant and quant.endswith("_groups") else 0
        if quant is None:
            self.y = torch.empty((rows, K), **bf16)
        else:
            t = torch.int8 if quant.startswith("i8") else torch.float8_e4m3fn
            self.q, self.q_scales = B.alloc_rmsnorm_quant(rows, K, self.q_group, t, device)

    def load(self, w, stream=None):
        """Real weights [N][K], quantised."""
        B.xnor_w4_quantize(w, self.d, self.packed, self.scales, self.zeros, stream)

    def forward(self, stream=None):
        """residual += x, out = norm(residual) times the weights."""
        if self.q is None:
            B.xnor_rmsnorm(self.x, self.residual, self.weight, self.eps, self.residual, self.y, None, stream)
        else:
            B.xnor_rmsnorm_quant(self.x, self.residual, self.weight, self.eps, self.q_group, self.residual, self.q,
                                 self.q_scales, None, stream)
        B.xnor_w4_matmul(self.y if self.q is None else self.q, self.q_scales, self.packed, self.scales, self.zeros,
                         self.d, self.out, stream)
        return self.out


class TokenAttention:
    """Buffers and calls of the attention in a decoder's layer, on bfloat16 rows between two TokenBlocks' products: norms
    and rotation of queries and keys, the new tokens into a cache in 4 bits, and attention over it.

    `seqs` sequences of up to `context` tokens each, in pages of `page` (tokens behind that are left out, and the next
    xnor_check_device says so); up to `rows` new tokens in a call, up to `most` of a sequence (0: any; a call of few takes
    longer then).  rot: rotated values of a head (None: all, 0: none)."""

    def __init__(self, rows, seqs, context, q_heads, kv_heads, dim, page=64, most=0, norm=True, rot=None, base=10000.0,
                 pairs=False, eps=1e-6, device="cuda"):
        cols = -(-context // page)
        self.q_heads, self.kv_heads, self.dim, self.most, self.pairs = q_heads, kv_heads, dim, most, pairs
        self.d = B.make_kv4_desc(seqs * cols, page, kv_heads, dim)
        self.cache = B.alloc_kv4(self.d, device)
        self.table = torch.arange(seqs * cols, dtype=torch.int32, device=device).view(seqs, cols)
        self.starts = torch.zeros((seqs + 1,), dtype=torch.int32, device=device)
        self.lens = torch.zeros((seqs,), dtype=torch.int32, device=device)
        rot = dim if rot is None else rot
        self.rope = B.make_rope(context, rot, base, device) if rot else None
        self.eps = eps if norm else None
        self.q_weight, self.k_weight = (torch.ones((dim,), dtype=torch.float32, device=device) if norm else None for _ in "qk")
        self.q = torch.empty((rows, q_heads, dim), dtype=torch.bfloat16, device=device)
        self.out = torch.empty((rows, q_heads * dim), dtype=torch.bfloat16, device=device)
        self.work = B.alloc_kv4_work(self.d, rows, q_heads, seqs, device)

    def grow(self, new):
        """The next forward() brings new[b] more tokens of sequence b (int32 on the device), in the sequences' order."""
        torch.cumsum(new, 0, dtype=torch.int32, out=self.starts[1:])
        self.lens += new

    def forward(self, qkv, stream=None):
        """qkv: rows [q_heads dim | kv_heads dim | kv_heads dim] of one product; gives rows [q_heads dim]."""
        rows, n, m = qkv.shape[0], self.q_heads, self.kv_heads
        q, k, v = (t.unflatten(1, (-1, self.dim)) for t in qkv.split([n * self.dim, m * self.dim, m * self.dim], 1))
        out = self.out[:rows]
        B.xnor_kv4_append(q, k, v, self.q_weight, self.k_weight, self.eps, self.rope, self.pairs, self.starts, self.lens,
                          self.table, self.d, self.q[:rows], self.cache, stream)
        B.xnor_kv4_attention(self.q[:rows], self.cache, self.starts, self.lens, self.table, self.d, self.dim ** -0.5,
                             self.most, out.unflatten(1, (n, self.dim)), None, self.work, stream)
        return out
