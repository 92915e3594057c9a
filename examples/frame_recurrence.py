"""Two ways of mixing frames over time in one block, trained with a trainable Mel layer by one optimiser, then run frame by frame as a stream.

    python examples/frame_recurrence.py

Clips of a few tones go through a Mel layer whose kernels and filters are parameters.  The block's queries and keys are normalised and rotated by their frames' positions before
linear attention mixes them; a gated recurrence beside it remembers channel by channel.  AdamW holds the moments of all of it, bfloat16 weights and the float32 kernels, in 8 bits, and
the trained network takes the frames one at a time with the two states in the place of the past.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from frame_model import DEVICE, SR, TONES, clips  # noqa: E402
from paper_1912_12055_amd import layers  # noqa: E402


class RecurrentFrameModel(torch.nn.Module):
    """Mel frames -> tokens -> linear attention and a gated recurrence, side by side -> a class for each frame."""

    def __init__(self, mels=40, n_fft=512, hop=256, width=128, heads=2, classes=TONES, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.width = heads, width
        self.mel = layers.MelSpectrogram(sr=SR, n_fft=n_fft, hop_length=hop, n_mels=mels, trainable_mel=True, trainable_STFT=True, device=DEVICE)
        self.frames_norm = layers.LayerNorm(mels, out_dtype=dtype, device=DEVICE)
        self.inwards = torch.nn.Linear(mels, width, device=DEVICE, dtype=dtype)
        self.projections = torch.nn.Linear(width, 6 * width, device=DEVICE, dtype=dtype)  # q, k, v; the recurrence's input and its two gates
        self.turn = layers.RotaryHeads(width // heads, base=1000.0, device=DEVICE)
        self.mix = layers.DecayAttention(heads, device=DEVICE)
        self.remember = layers.GatedRecurrence()
        self.norm = layers.LayerNorm(width, device=DEVICE)
        self.outwards = torch.nn.Linear(width, classes, device=DEVICE, dtype=dtype)

    def tokens(self, wave):
        """[B, T, mels] of waveforms [B, L]"""
        # (a trained filter may be negative between its neighbours' bins)
        return self.frames_norm(torch.log(self.mel(wave).clamp(min=1e-4)).transpose(1, 2))

    def _parts(self, x):
        q, k, v, x, forget, input = self.projections(x).chunk(6, -1)
        return (*(t.unflatten(-1, (self.heads, -1)) for t in (q, k, v)), x, forget + 2, input)

    def forward(self, tokens, lengths=None):
        """(logits [B, T, classes], (both states after the last frame))"""
        h = self.inwards(tokens)
        q, k, v, x, forget, input = self._parts(h)
        q, k = self.turn(q, k)
        mixed, s1 = self.mix(q, k, v, lengths=lengths, return_state=True)
        kept, s2 = self.remember(x, forget, input, lengths=lengths, return_state=True)
        return self.outwards(self.norm(h + mixed.flatten(-2) + kept)).float(), (s1, s2)

    def step(self, token, at, states):
        """logits [B, classes] of one new frame at positions `at` (int32 [B] on the GPU); the states are updated in place"""
        h = self.inwards(token)
        q, k, v, x, forget, input = self._parts(h)
        q, k = self.turn(q, k, positions=at)
        mixed = self.mix.step(q, k, v, states[0])
        kept = self.remember.step(x, forget, states[1], input)
        return self.outwards(self.norm(h + mixed.flatten(-2) + kept)).float()


def train(model, steps, batch=8, seed=0, bits=8, lr=2e-3):
    generator = torch.Generator(device=DEVICE).manual_seed(seed)
    transform = list(model.mel.parameters())
    network = [p for p in model.parameters() if not any(p is t for t in transform)]
    # (the transform starts as what it is meant to be: its kernels and filters move little)
    optimiser = layers.AdamW([dict(params=network, lr=lr), dict(params=transform, lr=1e-5, weight_decay=0.0)], bits=bits)
    losses = []
    for _ in range(steps):
        wave, lengths, tone = clips(batch, generator)
        tone = tone[:, : 1 + wave.shape[1] // model.mel.hop_length]
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
    logits, states = model(tokens[:, :prompt])
    at = torch.full((tokens.shape[0],), prompt, dtype=torch.int32, device=DEVICE)
    steps = []
    for t in range(prompt, tokens.shape[1]):
        steps.append(model.step(tokens[:, t], at, states))
        at += 1
    return torch.cat([logits, torch.stack(steps, 1)], 1)


def main():
    torch.manual_seed(0)
    model = RecurrentFrameModel()
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
