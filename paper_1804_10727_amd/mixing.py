"""Live signals whose rows are mixed over time: the streaming net makes feature rows of what comes in, every finished row is a token, and
two layers on top look back over the stream -- one attends to a window and the first tokens, one carries a decaying sum.  Rings and states
have a fixed size, as the net's rolling buffers do: memory does not grow with the signal.

    python -m paper_1804_10727_amd.mixing [--streams 64] [--samples 4000] [--segment 16] [--window 256] [--few-bits]

In few bits the products take 8-bit weights, the rings hold 4-bit blocks, and a gated recurrence per channel takes the place of the decaying sum: 37,800
bytes for a stream with the values above, where the other form has 315,400 in float32 and 174,088 in bfloat16.

The mixers' weights are random: what they show is how the calls go together.  GatedReadout on top of rows like theirs is trained.
"""
from __future__ import annotations

import argparse
import time

from .tokens import (decay_attend, gate_scan, gate_scan_recorded, nibble_append, nibble_attend, nibble_ring, norm_rotate, project_rows, quantize_rows,
                     rotary_frequencies, window_attend)


class _Mixer:
    """What mixers of `n_streams` streams of rows have in common: norms and rotation of queries and keys, and where each stream stands."""

    def __init__(self, n_streams, heads, kv_heads, dim, window, sinks, dtype, device):
        import torch
        self.heads, self.kv_heads, self.dim, self.window, self.sinks = heads, kv_heads, dim, window, sinks
        self.dtype = torch.float32 if dtype is None else dtype
        self.frequencies, self.amplitude = rotary_frequencies(dim, device=device)
        self.starts = torch.zeros(n_streams, dtype=torch.int64, device=device)

    def _norms(self, g, device):
        import torch
        self.q_weight, self.k_weight = (1 + 0.1 * torch.randn(self.dim, generator=g).to(device) for _ in range(2))

    def state_bytes(self):
        """Per stream, whatever its length."""
        return sum(t[0].numel() * t.element_size() for t in (*self.rings, self.state, self.starts))

    def _heads(self, packed):
        return packed.unflatten(1, (-1, self.dim)).split([self.heads, self.kv_heads, self.kv_heads], 1)

    def _segments(self, x, counts):
        """How many rows of each stream, where each row stands in its stream, and the segments as the operators take them."""
        import torch
        streams = self.starts.numel()
        # (on the GPU nothing would refuse wrong counts: positions are laid out for so many rows)
        if counts is None:
            if x.shape[0] % streams:
                raise ValueError(f"{x.shape[0]} rows are not as many of each of {streams} streams")
            n = torch.full_like(self.starts, x.shape[0] // streams)
        else:
            counts = torch.as_tensor(counts)
            if counts.dtype.is_floating_point or counts.shape != (streams,) or int(counts.min()) < 0 or int(counts.sum()) != x.shape[0]:
                raise ValueError(f"{x.shape[0]} rows of {streams} streams, {counts.tolist()} of each")
            n = counts.to(x.device, torch.int64)
        ends = n.cumsum(0)
        segments = {} if counts is None else dict(offsets=torch.cat([ends.new_zeros(1), ends]), max_tokens=int(counts.max()))
        positions = torch.arange(x.shape[0], device=x.device) + torch.repeat_interleave(self.starts - ends + n, n, output_size=x.shape[0])
        return n, positions, segments


class TokenMixer(_Mixer):
    """The two layers for `n_streams` streams of rows of `channels` values; push() takes what is new of each."""

    def __init__(self, channels, n_streams, heads=4, kv_heads=2, dim=64, window=256, sinks=4, room=16, dtype=None, device="cuda:0", seed=0):
        import torch
        super().__init__(n_streams, heads, kv_heads, dim, window, sinks, dtype, device)
        g = torch.Generator().manual_seed(seed)
        dtype, width = self.dtype, (heads + 2 * kv_heads) * dim

        def weights(rows, cols):
            return (torch.randn(rows, cols, generator=g) / rows ** 0.5).to(device, dtype)
        self.project, self.back = ([weights(*s) for _ in range(2)] for s in ((channels, width), (heads * dim, channels)))
        self._norms(g, device)
        self.log_decay = -torch.exp2(-torch.arange(3, 3 + kv_heads, dtype=torch.float32)).to(device)
        # room for a segment beside the window: its tokens then go to the ring in the launch that attends over them
        self.rings = [torch.zeros(n_streams, sinks + window + room, kv_heads, dim, dtype=dtype, device=device) for _ in range(2)]
        self.state = torch.zeros(n_streams, kv_heads, dim, dim, device=device)

    def _split(self, x, layer):
        return self._heads(x @ self.project[layer])

    def push(self, x, counts=None):
        """x: the new rows of all streams behind each other, [rows][channels]; counts: how many of each stream (None: the same of all)."""
        n, positions, segments = self._segments(x, counts)
        q, k, v = self._split(x, 0)
        norm_rotate(q, k, positions, self.frequencies, amplitude=self.amplitude, q_weight=self.q_weight, k_weight=self.k_weight, q_out=q, k_out=k)
        seen = window_attend(q, k, v, *self.rings, self.starts, window=self.window, sinks=self.sinks, **segments)
        x = x + seen.flatten(1) @ self.back[0]
        q, k, v = self._split(x, 1)
        carried = decay_attend(q, k, v, self.log_decay, self.state, self.state, **segments)
        self.starts += n
        return x + carried.flatten(1) @ self.back[1]


class FewBitsMixer(_Mixer):
    """The same for few bits: 8-bit products, rings of 4-bit blocks that have room for `room` rows of a stream beside a window, and on top of them a recurrence
    whose gates its own rows give."""

    def __init__(self, channels, n_streams, heads=4, kv_heads=2, dim=64, window=256, sinks=4, room=16, dtype=None, device="cuda:0", seed=0):
        import torch
        super().__init__(n_streams, heads, kv_heads, dim, window, sinks, dtype, device)
        g = torch.Generator().manual_seed(seed)
        # as rows of outputs: queries, keys and values; back from the heads; gates and what they let in
        shapes = (((heads + 2 * kv_heads) * dim, channels), (channels, heads * dim), (2 * channels, channels))
        self.weights = [quantize_rows((torch.randn(*s, generator=g) / s[1] ** 0.5).to(device)) for s in shapes]
        self.gate_bias = torch.cat([torch.linspace(0.0, 6.0, channels), torch.zeros(channels)]).to(device)
        self._norms(g, device)
        self.room, self.rings = room, nibble_ring(n_streams, sinks + window + room, kv_heads, dim, device)
        self.state = torch.zeros(n_streams, channels, device=device)

    def push(self, x, counts=None):
        """As TokenMixer.push; at most room + 1 rows of a stream at a time."""
        n, positions, segments = self._segments(x, counts)
        if segments.get("max_tokens", x.shape[0] // len(self.starts)) > self.room + 1:
            raise ValueError(f"rings with room for {self.room} rows beside a window take pieces of up to {self.room + 1}")
        q, k, v = self._heads(project_rows(x, *self.weights[0]))
        norm_rotate(q, k[:, :0], positions, self.frequencies, amplitude=self.amplitude, q_weight=self.q_weight, q_out=q, k_out=k[:, :0])
        nibble_append(k, v, self.rings, self.starts, sinks=self.sinks, frequencies=self.frequencies, amplitude=self.amplitude, k_weight=self.k_weight, **segments)
        seen = nibble_attend(q, self.rings, self.starts, window=self.window, sinks=self.sinks, **segments)
        x = x + project_rows(seen.flatten(1), *self.weights[1])
        gates, new = project_rows(x, *self.weights[2], bias=self.gate_bias).chunk(2, 1)
        self.starts += n
        return x + gate_scan(new, gates, self.state, self.state, **segments)


class GatedReadout:
    """Class scores from the rows of many signals, on a gated recurrence that is trained for it: gates and values are linear in a row, scores in the state that a
    signal ends with.  parameters() for an optimizer; loss() records through gate_scan_recorded."""

    def __init__(self, channels, classes, hidden=64, device="cuda:0", seed=0):
        import torch
        g = torch.Generator().manual_seed(seed)
        self.into = (torch.randn(channels, 2 * hidden, generator=g) / channels ** 0.5).to(device).requires_grad_()
        self.bias = torch.cat([torch.linspace(0.0, 4.0, hidden), torch.zeros(hidden)]).to(device).requires_grad_()
        self.out = (torch.randn(hidden, classes, generator=g) / hidden ** 0.5).to(device).requires_grad_()

    def parameters(self):
        return [self.into, self.bias, self.out]

    def scores(self, rows, offsets, max_tokens):
        """rows: float32 [row][channel] of all signals behind each other; [signal][class]."""
        gates, new = (rows @ self.into + self.bias).chunk(2, 1)
        return gate_scan_recorded(new, gates, offsets=offsets, max_tokens=max_tokens)[1] @ self.out

    def loss(self, rows, offsets, max_tokens, labels):
        import torch
        return torch.nn.functional.cross_entropy(self.scores(rows, offsets, max_tokens), labels)


def listen(wl, segment, mixer):
    """The workload's signals pushed `segment` samples at a time through the net and the mixer: yields the rows that came out of each push,
    [streams][rows][channels]."""
    from . import Streams, net_from_workload
    from .binding import input_tensor
    net = net_from_workload(wl)
    st = Streams(net, wl["streams"], max_seg_rows=segment)
    x = input_tensor(wl)
    for at in range(0, x.shape[1], segment):
        st.push_segment(x[:, at:at + segment].contiguous())
        rows, _, counts = st.read_outputs(segment)
        n = int(counts[0])                         # (all streams are pushed together)
        if n:
            tokens = rows[:, :n].flatten(2).to(mixer.dtype).flatten(0, 1)
            yield mixer.push(tokens).unflatten(0, (wl["streams"], n))
    st.close()
    net.destroy()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--streams", type=int, default=64)
    ap.add_argument("--samples", type=int, default=4000)
    ap.add_argument("--segment", type=int, default=16)
    ap.add_argument("--window", type=int, default=256)
    ap.add_argument("--few-bits", action="store_true")
    args = ap.parse_args()
    import torch
    import workloads
    wl = workloads.make(2, streams=args.streams, length=args.samples)
    for run in range(2):                           # (the first one loads)
        mixer = (FewBitsMixer if args.few_bits else TokenMixer)(wl["layers"][-1]["c_out"], args.streams, window=args.window, room=args.segment)
        torch.cuda.synchronize()
        began = time.perf_counter()
        rows = [r.shape[1] for r in listen(wl, args.segment, mixer)]
        torch.cuda.synchronize()
        took = time.perf_counter() - began
    pushes = -(-args.samples // args.segment)
    print(f"{args.streams} signals of {args.samples} samples, {args.segment} at a time: {sum(rows)} rows of each mixed over the last {args.window}; "
          f"{1e6 * took / pushes:.0f} us per push, {mixer.state_bytes()} bytes of rings and states per stream")


if __name__ == "__main__":
    main()
