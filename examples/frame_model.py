"""A network on the transforms' frames: trained on whole clips, then run frame by frame as a stream.

    python examples/frame_model.py

Clips of a few tones, most of them shorter than the batch, go through a Mel layer; their frames are normalised as they lie, mixed over time
by linear attention with a decay for each head, and every frame is told which of the tones it heard last.  What the block's second norm needs in its
backward pass is kept in 8 bits.  The trained network then takes the same frames one at a time, with a state in the place of the past.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1912_12055_amd import layers  # noqa: E402

DEVICE = "cuda:0"
SR, HOP, TONES = 16000, 256, 12


class FrameModel(torch.nn.Module):
    """Mel frames -> tokens -> one block of linear attention -> a class for each frame."""

    def __init__(self, mels=80, width=256, heads=4, classes=TONES, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.dtype = heads, dtype
        self.mel = layers.MelSpectrogram(sr=SR, n_fft=1024, hop_length=HOP, n_mels=mels, device=DEVICE)
        self.frames_norm = layers.LayerNorm(mels, out_dtype=dtype, device=DEVICE)
        self.inwards = torch.nn.Linear(mels, width, device=DEVICE, dtype=dtype)
        self.qkv = torch.nn.Linear(width, 3 * width, device=DEVICE, dtype=dtype)
        self.mix = layers.DecayAttention(heads, device=DEVICE)
        self.norm = layers.LayerNorm(width, kept_bits=8, device=DEVICE)
        self.outwards = torch.nn.Linear(width, classes, device=DEVICE, dtype=dtype)

    def tokens(self, wave):
        """[B, T, mels] of waveforms [B, L]: the logarithm of their Mel frames, normalised without a transposed copy"""
        with torch.no_grad():
            spec = torch.log(self.mel(wave) + 1e-6)
        return self.frames_norm(spec.transpose(1, 2))

    def _heads(self, x):
        return self.qkv(x).unflatten(-1, (3, self.heads, -1)).unbind(-3)

    def forward(self, tokens, lengths=None, state=None):
        """(logits [B, T, classes], state after the last frame)"""
        x = self.inwards(tokens)
        mixed, state = self.mix(*self._heads(x), state=state, lengths=lengths, return_state=True)
        return self.outwards(self.norm(x + mixed.flatten(-2))).float(), state

    def step(self, token, state):
        """logits [B, classes] of one new frame; `state` is updated in place"""
        x = self.inwards(token)
        mixed = self.mix.step(*self._heads(x), state)
        return self.outwards(self.norm(x + mixed.flatten(-2))).float()


def clips(batch, generator, seconds=2.0):
    """(waveforms [B, L], frames of each clip [B], the tone of each frame [B, T])"""
    length = int(seconds * SR)
    frames = 1 + length // HOP
    t = torch.arange(length, device=DEVICE) / SR
    parts = 4
    tone = torch.randint(0, TONES, (batch, parts), device=DEVICE, generator=generator)
    part = torch.arange(length, device=DEVICE) * parts // length
    hz = 220 * 2 ** (tone / 12)
    wave = 0.3 * torch.sin(2 * torch.pi * hz[:, part] * t) + 0.05 * torch.randn(batch, length, device=DEVICE, generator=generator)
    lengths = (frames * (0.5 + 0.5 * torch.rand(batch, device=DEVICE, generator=generator))).to(torch.int32)
    lengths[0] = frames
    at = (torch.arange(frames, device=DEVICE) * HOP).clamp(max=length - 1)
    return wave, lengths, tone[:, part[at]]


def train(model, steps, batch=16, seed=0):
    generator = torch.Generator(device=DEVICE).manual_seed(seed)
    optimiser = torch.optim.Adam(model.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        wave, lengths, tone = clips(batch, generator)
        logits, _ = model(model.tokens(wave), lengths=lengths)
        here = torch.arange(tone.shape[1], device=DEVICE) < lengths[:, None]
        loss = torch.nn.functional.cross_entropy(logits[here], tone[here])
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


@torch.no_grad()
def stream(model, tokens, prompt):
    """logits of all frames, the first `prompt` of them at once and the others one at a time"""
    logits, state = model(tokens[:, :prompt])
    steps = [model.step(tokens[:, t], state) for t in range(prompt, tokens.shape[1])]
    return torch.cat([logits, torch.stack(steps, 1)], 1)


def main():
    torch.manual_seed(0)
    model = FrameModel()
    losses = train(model, 60)
    print("loss", " ".join(f"{v:.3f}" for v in losses[::10]), f"{losses[-1]:.3f}")
    with torch.no_grad():
        wave, _, tone = clips(4, torch.Generator(device=DEVICE).manual_seed(99))
        tokens = model.tokens(wave)
        whole, _ = model(tokens)
        one_by_one = stream(model, tokens, prompt=40)
    print(f"frames told right: {float((whole.argmax(-1) == tone).float().mean()):.2f}; "
          f"frame by frame against the whole: {float((one_by_one - whole).norm() / whole.norm()):.4f}")


if __name__ == "__main__":
    main()
